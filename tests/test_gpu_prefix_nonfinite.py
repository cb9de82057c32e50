"""Values that are not finite in prefix-shared and verification calls: the rows that see them have what the formula gives, and
beams that share a unit with them have theirs."""

import math

import numpy as np
import pytest
import torch

from oracle.cached_ops import chunk_attention
from paper_2509_00195_amd import (tts_build_prefix_meta, tts_build_verify_meta, tts_prefix_decode_attn,
                                  tts_prefix_decode_attn_noalloc, tts_prefix_decode_workspace_size, tts_prefix_verify_attn)
from tests._cached import BS, DEV, KINDS, Cache, desc_of, queries, reference

pytestmark = pytest.mark.gpu


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _tree(kind, hkv, d, beams, share, spread, seed, requests=1, least=1):
    """Beams of each request share `share` blocks and have `least` to `spread` tokens more."""
    rng = np.random.default_rng(seed)
    c = Cache(kind, hkv, d, 16 * share + rng.integers(least, spread + 1, beams), rng)
    per = beams // requests
    for r in range(requests):
        c.tables[r * per:(r + 1) * per, :share] = c.tables[r * per, :share]
    return c, np.arange(0, beams + 1, per, dtype=np.int32)


def _bad_value(c, b, token, head, dim, x=np.nan):
    """Makes a value (4-bit caches: its group of 32 dims) of a beam's token NaN, or x."""
    p, slot = c.tables[b, token // BS], token % BS
    if c.kind == "mx4":
        c.v[p, head, BS * c.d // 2 + dim // 32 * BS + slot] = 255
    elif c.kind == "fp8":
        c.v[p, head, dim, slot] = 0x7F
    elif c.kind == "bf16":
        c.v[p, head, dim, slot] = {math.inf: 0x7F80, -math.inf: 0xFF80}.get(x, 0x7FC0)
    else:
        c.v[p, head, dim, slot] = x


def _call(c, hq, offs, q, q_len=1, lens=None, noalloc=False):
    """Metadata for `lens` (default: the beams' lengths), the call at their lengths."""
    desc = desc_of(c.kind, hq, c.hkv, c.d)
    built = c.lens if lens is None else lens
    meta = tts_build_verify_meta(offs, c.tables, built, q_len, BS, c.nb, desc=desc) if q_len > 1 else \
        tts_build_prefix_meta(offs, c.tables, built, BS, c.nb, desc=desc)
    out = torch.full(q.shape, 5.0, device=DEV)
    args = (desc, meta, q, *c.device(), _up(c.tables), c.tables.shape[1], _up(c.lens), c.nb, out)
    if noalloc:
        tts_prefix_decode_attn_noalloc(*args)
    else:
        size = tts_prefix_decode_workspace_size(desc, meta)
        call = tts_prefix_verify_attn if q_len > 1 else tts_prefix_decode_attn
        call(*args, torch.empty(size, dtype=torch.uint8, device=DEV), size)
    return out.cpu().numpy()


def _check(c, clean, b, got, qv):
    """Rows [n][hq][d] of beam b's last n tokens."""
    k, v = c.dense(b)
    with np.errstate(invalid="ignore"):
        want = chunk_attention(qv, k, v, len(qv), 1.0 / math.sqrt(c.d))[0]
    _, tol = reference(clean, b, qv)
    for f in (np.isposinf, np.isneginf, np.isnan):
        assert (f(got) == f(want)).all(), b
    keep = np.isfinite(want)
    assert (np.abs(got - np.where(keep, want, 0)) <= tol)[keep].all(), b


SHAPES = [(64, 59, 16, 2, 64, 1), (64, 9, 8, 2, 64, 4), (96, 20, 28, 4, 128, 1), (24, 3, 3, 1, 64, 2)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beams,share,hq,hkv,d,requests", SHAPES)
@pytest.mark.parametrize("spread", [1, 40])
def test_a_beam_does_not_reach_the_others(kind, beams, share, hq, hkv, d, requests, spread):
    make = lambda: _tree(kind, hkv, d, beams, share, spread, 0, requests)  # noqa: E731
    (c, offs), (clean, _) = make(), make()
    for b in (1, beams // 2, beams - 1):
        _bad_value(c, b, 16 * share, hkv - 1, 5)
    q, qv = queries(kind, (beams, hq, d), np.random.default_rng(1))
    got = _call(c, hq, offs, q)
    bad = [b for b in range(beams) if np.isnan(got[b]).any()]
    assert bad == [1, beams // 2, beams - 1]
    for b in (0, 1, 2, beams // 2 - 1, beams // 2, beams // 2 + 1, beams - 2, beams - 1):
        _check(c, clean, b, got[b][None], qv[b][None])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_infinities_of_both_signs(kind):
    make = lambda: _tree(kind, 2, 128, 64, 20, 40, 2)  # noqa: E731
    (c, offs), (clean, _) = make(), make()
    for b, dim, x in ((3, 7, math.inf), (4, 7, -math.inf), (4, 90, math.inf), (40, 90, math.inf)):
        _bad_value(c, b, 320, 1, dim, x)
    _bad_value(c, 40, 319, 1, 90, -math.inf)  # in a shared block: every beam's; beam 40 sees both signs
    q, qv = queries(kind, (64, 8, 128), np.random.default_rng(3))
    for noalloc in (False, True):
        got = _call(c, 8, offs, q, noalloc=noalloc)
        for b in (0, 2, 3, 4, 5, 39, 40, 41):
            _check(c, clean, b, got[b][None], qv[b][None])


@pytest.mark.parametrize("kind", KINDS)
def test_growth_and_scales(kind):
    """A block that a beam gained after its metadata was built; fp8: a V scale that is not finite."""
    make = lambda: _tree(kind, 2, 64, 48, 9, 40, 4)  # noqa: E731
    (c, offs), (clean, _) = make(), make()
    built = np.full(48, 16 * 9 + 1, np.int32)
    grown = [b for b in range(48) if c.lens[b] > 16 * 10][::3]
    for b in grown:
        if kind == "fp8":
            c.vs[c.tables[b, 10]] = np.inf
        else:
            _bad_value(c, b, 160, 0, 33)
    q, qv = queries(kind, (48, 8, 64), np.random.default_rng(5))
    got = _call(c, 8, offs, q, lens=built)
    for b in range(48):
        if b in grown:
            assert not np.isfinite(got[b]).all()
        else:
            _check(c, clean, b, got[b][None], qv[b][None])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beams,share,hq,hkv,d", [(16, 9, 6, 2, 64), (64, 9, 8, 2, 64), (32, 20, 28, 4, 128)])
def test_verification(kind, beams, share, hq, hkv, d):
    """A token's value reaches the queries of that token and later ones of its beam alone."""
    make = lambda: _tree(kind, hkv, d, beams, share, 40, 6, least=4)  # noqa: E731
    (c, offs), (clean, _) = make(), make()
    for b, back in ((1, 1), (beams // 2, 2), (beams - 1, 1)):
        _bad_value(c, b, int(c.lens[b]) - back, 0, 5)
    q, qv = queries(kind, (beams, 3, hq, d), np.random.default_rng(7))
    got = _call(c, hq, offs, q, 3)
    bad = [(b, i) for b in range(beams) for i in range(3) if np.isnan(got[b, i]).any()]
    assert bad == [(1, 2), (beams // 2, 1), (beams // 2, 2), (beams - 1, 2)]
    for b in (0, 1, 2, beams // 2 - 1, beams // 2, beams - 2, beams - 1):
        _check(c, clean, b, got[b], qv[b])
