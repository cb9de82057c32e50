"""NaN keys and queries through calls that join partial states: split paged calls and prefix-shared ones."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import (tts_build_prefix_meta, tts_build_verify_meta, tts_paged_decode_attn,
                                  tts_paged_decode_workspace_size, tts_prefix_decode_attn,
                                  tts_prefix_decode_workspace_size, tts_prefix_verify_attn)
from tests._cached import BS, DEV, KINDS, Cache, desc_of, queries, reference

pytestmark = pytest.mark.gpu


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _nan_key(c, block, head, slot):
    """Makes the key of a token NaN."""
    if c.kind == "mx4":
        c.k[block, head, BS * c.d // 2 + slot * c.d // 32] = 255
    else:
        c.k[block, head, slot, 5] = {"f32": np.nan, "bf16": 0x7FC0, "fp8": 0x7F}[c.kind]


def _paged(c, q, out, hq, most):
    desc = desc_of(c.kind, hq, c.hkv, c.d)
    size = tts_paged_decode_workspace_size(desc, len(c.lens), most)
    assert size > 0  # split
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    tts_paged_decode_attn(desc, len(c.lens), q, *c.device(), _up(c.tables), c.tables.shape[1], _up(c.lens), most, c.nb, out, ws,
                          size)
    return out.cpu().numpy()


def _shared(c, q, out, hq, offs, q_len=1):
    desc = desc_of(c.kind, hq, c.hkv, c.d)
    build = lambda *a: tts_build_verify_meta(offs, c.tables, c.lens, q_len, *a, desc=desc) if q_len > 1 else \
        tts_build_prefix_meta(offs, c.tables, c.lens, *a, desc=desc)  # noqa: E731
    meta = build(BS, c.nb)
    size = tts_prefix_decode_workspace_size(desc, meta)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    call = tts_prefix_verify_attn if q_len > 1 else tts_prefix_decode_attn
    call(desc, meta, q, *c.device(), _up(c.tables), c.tables.shape[1], _up(c.lens), c.nb, out, ws, size)
    return out.cpu().numpy()


def _check(c, clean, got, qv, nan):
    """Rows where `nan` [sequences][heads] says so are NaN, the others those of the clean cache."""
    for b in range(len(c.lens)):
        assert np.isnan(got[b][nan[b]]).all(), b
        if c.lens[b] == 0:
            assert (got[b] == 0).all()
            continue
        want, tol = reference(clean, b, qv[b][None])
        assert (np.abs(got[b] - want[0]) <= tol[0])[~nan[b]].all(), b


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(6, 2), (36, 2)])
def test_nan_keys_in_split_calls(kind, hq, hkv):
    """One non-empty split that holds the key, and one of several."""
    make = lambda: Cache(kind, hkv, 64, [40, 0, 700, 40, 1500], np.random.default_rng(0), cols=256)  # noqa: E731
    c, clean = make(), make()
    q, qv = queries(kind, (5, hq, 64), np.random.default_rng(1))
    nan = np.zeros((5, hq), bool)
    for b, token, head in ((0, 21, 0), (2, 699, 1), (4, 0, 1)):
        _nan_key(c, c.tables[b, token // BS], head, token % BS)
        nan[b, head * hq // 2:(head + 1) * hq // 2] = True
    _check(c, clean, _paged(c, q, torch.zeros((5, hq, 64), device=DEV), hq, 4096), qv, nan)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(6, 2), (36, 2)])
def test_nan_queries_in_split_calls(kind, hq, hkv):
    c = Cache(kind, hkv, 64, [40, 0, 700, 1], np.random.default_rng(2), cols=256)
    q, qv = queries(kind, (4, hq, 64), np.random.default_rng(3))
    nan = np.zeros((4, hq), bool)
    for b, h in ((0, 1), (1, 2), (2, hq - 1), (3, 0)):
        q[b, h, 7] = np.nan
        nan[b, h] = c.lens[b] > 0  # (a sequence without tokens has zero rows)
    _check(c, c, _paged(c, q, torch.zeros((4, hq, 64), device=DEV), hq, 4096), qv, nan)


def _tree(kind, beams, share, lo, hi, seed):
    """Beams of one request that share `share` blocks."""
    rng = np.random.default_rng(seed)
    c = Cache(kind, 2, 64, rng.integers(lo, hi, beams), rng)
    c.tables[:, :share] = c.tables[0, :share]
    return c


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beams,share,hq", [(12, 9, 6), (64, 59, 16), (160, 59, 16)])
def test_nan_queries_of_some_beams(kind, beams, share, hq):
    """Narrow and wide units (whole and in halves): a beam's rows through all of its states."""
    c = _tree(kind, beams, share, 16 * share + 10, 16 * share + 90, 4)
    offs = np.array([0, beams], np.int32)
    q, qv = queries(kind, (beams, hq, 64), np.random.default_rng(5))
    nan = np.zeros((beams, hq), bool)
    for b, h in ((0, 0), (beams // 2, 3), (beams - 1, hq - 1)):
        q[b, h, 7] = np.nan
        nan[b, h] = True
    got = _shared(c, q, torch.zeros((beams, hq, 64), device=DEV), hq, offs)
    for b in range(beams):
        assert np.isnan(got[b][nan[b]]).all() and np.isfinite(got[b][~nan[b]]).all(), b
    keep = [0, 1, beams // 2, beams - 1]
    for b in keep:
        want, tol = reference(c, b, qv[b][None])
        assert (np.abs(got[b] - want[0]) <= tol[0])[~nan[b]].all(), b


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beams,share,hq", [(12, 9, 6), (64, 59, 16)])
def test_nan_key_in_the_shared_prefix_alone(kind, beams, share, hq):
    """Every beam ends with the shared blocks: its only states hold the key."""
    c = _tree(kind, beams, share, 16 * share, 16 * share + 1, 6)
    _nan_key(c, c.tables[0, 3], 1, 2)
    q, _ = queries(kind, (beams, hq, 64), np.random.default_rng(7))
    got = _shared(c, q, torch.zeros((beams, hq, 64), device=DEV), hq, np.array([0, beams], np.int32))
    assert np.isnan(got[:, hq // 2:]).all() and np.isfinite(got[:, :hq // 2]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_nan_queries_in_verification(kind):
    """A NaN query of one of a beam's tokens: its row, and no other token's."""
    c = _tree(kind, 7, 5, 90, 150, 8)
    q, qv = queries(kind, (7, 3, 6, 64), np.random.default_rng(9))
    nan = np.zeros((7, 3, 6), bool)
    for at in ((0, 0, 1), (3, 2, 5), (6, 1, 0)):
        q[at][7] = np.nan
        nan[at] = True
    got = _shared(c, q, torch.zeros((7, 3, 6, 64), device=DEV), 6, np.array([0, 7], np.int32), 3)
    assert np.isnan(got[nan]).all()
    for b in range(7):
        qb = np.where(nan[b][..., None], 0.0, qv[b])
        want, tol = reference(c, b, qb)
        assert (np.abs(got[b] - want) <= tol)[~nan[b]].all(), b


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv", [(6, 2), (36, 2)])
@pytest.mark.parametrize("gain", [1.0, 2.5, 6.0])
def test_infinite_values_in_split_calls(kind, hq, hkv, gain):
    """An infinite value makes its dim infinite and leaves the others, in rows of small and large sums."""
    make = lambda: Cache(kind, hkv, 64, [40, 700], np.random.default_rng(10), cols=256, gain=gain)  # noqa: E731
    c, clean = make(), make()
    for b, token in ((0, 3), (1, 650)):
        c.v[c.tables[b, token // BS], 1, 9, token % BS] = np.inf if kind == "f32" else 0x7F80
    q, qv = queries(kind, (2, hq, 64), np.random.default_rng(11), gain)
    got = _paged(c, q, torch.zeros((2, hq, 64), device=DEV), hq, 4096)
    for b in range(2):
        want, tol = reference(clean, b, qv[b][None])
        # (a probability below fp32's least normal, 2^-126 of the largest, may be held as 0, and 0 x inf is NaN)
        score = clean.dense(b)[0][1] @ qv[b, hq // 2:].T / 8.0
        seen = score[3 if b == 0 else 650] - score.max(0) > -125 * np.log(2)
        assert np.isposinf(got[b, hq // 2:, 9][seen]).all() and not np.isfinite(got[b, hq // 2:, 9]).any()
        got[b, hq // 2:, 9] = want[0, hq // 2:, 9]
        assert (np.abs(got[b] - want[0]) <= tol[0]).all()
