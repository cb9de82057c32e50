"""Ragged prefill attention against 64 bits."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import tts_paged_prefill_attn, tts_paged_prefill_workspace_size
from tests._cached import BS, DEV, KINDS, Cache, close, desc_of, queries, reference

pytestmark = pytest.mark.gpu


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _dtype(kind, out_t):
    return torch.float32 if out_t == "f32" else torch.bfloat16


def _call(c, desc, new, q, out, lens=None, tables=None, most=None, total=None, caches=None, nb=None, stream=None):
    lens = c.lens if lens is None else np.asarray(lens, np.int32)
    t = c.tables if tables is None else tables
    most = int(max(lens.max(), 1)) if most is None else most
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    total = int(q.shape[0]) if total is None else total
    size = tts_paged_prefill_workspace_size(desc, len(lens), total, most)
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device=DEV)
    tts_paged_prefill_attn(desc, len(lens), total, _up(offs), q, *(caches or c.device()), _up(t), t.shape[1], _up(lens), most,
                           nb or c.nb, out, ws, size, stream)
    torch.cuda.synchronize()
    return size


def _check(c, new, out, qv, rounded, skip=()):
    at = 0
    for b, n in enumerate(new):
        if n and b not in skip:
            want, tol = reference(c, b, qv[at:at + n])
            close(out[at:at + n], want, tol, rounded)
        at += n


RAGGED = ([1, 40, 16, 17, 129, 64, 300, 31, 90], [1, 40, 1, 16, 0, 33, 77, 2, 65])  # lengths, new tokens


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (15, 5, 64), (28, 4, 128), (3, 3, 128), (34, 2, 64)])
@pytest.mark.parametrize("out_t", ["f32", "bf16"])
def test_ragged_chunks(kind, hq, hkv, d, out_t):
    """Chunks from nothing to the whole sequence; unused slots and blocks hold NaN; rows behind the last are left."""
    rng = np.random.default_rng(0)
    lens, new = RAGGED
    c = Cache(kind, hkv, d, lens, rng)
    c.poison()
    total, pad = sum(new), 6
    q, qv = queries(kind, (total + pad, hq, d), rng, 2.0)
    out = torch.full((total + pad, hq, d), 5.0, dtype=_dtype(kind, out_t), device=DEV)
    _call(c, desc_of(kind, hq, hkv, d, out_t), new, q, out)
    assert (out[total:] == 5).all()
    _check(c, new, out, qv, out_t == "bf16")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (6, 2, 64)])
def test_few_rows_over_many_tokens(kind, hq, hkv, d):
    """Split over the tokens and joined; padded rows and unequal lengths (some splits see nothing)."""
    rng = np.random.default_rng(1)
    lens, new = [3000, 20, 1100, 0, 257], [5, 20, 1, 3, 2]
    c = Cache(kind, hkv, d, lens, rng)
    c.poison()
    total = sum(new)
    q, qv = queries(kind, (total + 4, hq, d), rng)
    out = torch.full((total + 4, hq, d), 5.0, device=DEV)
    assert _call(c, desc_of(kind, hq, hkv, d), new, q, out) > 0
    assert (out[total:] == 5).all() and (out[26:29] == 0).all()
    _check(c, new, out, qv, False, skip=(3,))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("split", [False, True])
def test_hidden_infinities_and_nan(kind, split):
    """Values (and keys) that are not finite at a token reach the rows of later queries and no others."""
    rng = np.random.default_rng(2)
    n, bad = (130, 71) if not split else (130, 1271)
    length = n if not split else 1330
    c = Cache(kind, 2, 64, [length], rng)
    p, slot = c.tables[0, bad // BS], bad % BS
    clean = c.dense(0)
    if kind == "mx4":  # one V group of a head
        c.v[p, 1, BS * 32 + slot] = 255
    elif kind == "fp8":
        c.v[p, 1, 3, slot] = 0x7F
    else:
        c.v[p, 1, 3, slot] = 0x7F80 if kind == "bf16" else np.inf
    q, qv = queries(kind, (n, 6, 64), rng)
    out = torch.zeros((n, 6, 64), device=DEV)
    used = _call(c, desc_of(kind, 6, 2, 64), [n], q, out)
    assert (used > 0) == split
    got = out.cpu().numpy()
    first = bad - (length - n)
    dims = slice(0, 32) if kind == "mx4" else slice(3, 4)
    assert not np.isfinite(got[first:, 3:, dims]).any()
    keep = got.copy()
    keep[first:, 3:, dims] = 0
    assert np.isfinite(keep).all()
    c.dense = lambda b, m=None: clean
    want, tol = reference(c, 0, qv)
    err = np.abs(got - want) <= tol
    err[first:, 3:, dims] = True
    assert err.all()
    # a key that is not finite: NaN rows of its head from its token on
    c2 = Cache(kind, 2, 64, [length], np.random.default_rng(3))
    if kind == "mx4":
        c2.k[c2.tables[0, bad // BS], 0, BS * 32 + 2 * slot] = 255
    else:
        c2.k[c2.tables[0, bad // BS], 0, slot, 5] = {"f32": np.nan, "bf16": 0x7FC0, "fp8": 0x7F}[kind]
    _call(c2, desc_of(kind, 6, 2, 64), [n], q, out)
    got = out.cpu().numpy()
    assert np.isnan(got[first:, :3]).all() and np.isfinite(got[:first]).all() and np.isfinite(got[:, 3:]).all()


def test_fp8_scale_of_a_hidden_block():
    """An infinite V scale: the rows that see the block, whole, and no others."""
    rng = np.random.default_rng(4)
    c = Cache("fp8", 1, 128, [100], rng)
    c.vs[c.tables[0, 4]] = np.inf
    q, qv = queries("fp8", (100, 4, 128), rng)
    out = torch.zeros((100, 4, 128), device=DEV)
    _call(c, desc_of("fp8", 4, 1, 128), [100], q, out)
    got = out.cpu().numpy()
    assert not np.isfinite(got[64:]).any() and np.isfinite(got[:64]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("most", [130, 1300])
def test_device_side_errors(kind, most):
    """Idle, too short, too long for the bound, too long for the table, and bad block ids; neighbours as ever. With
    max_seq_len 1300 the rows are split and joined."""
    rng = np.random.default_rng(5)
    lens = [40, 0, 5, 131 if most == 130 else 1301, 100, 128, 100]
    new = [10, 4, 9, 3, 60, 7, 60]
    c = Cache(kind, 2, 64, lens, rng, cols=most // BS + 1)
    q, qv = queries(kind, (sum(new), 4, 64), rng)
    out = torch.full((sum(new), 4, 64), 5.0, device=DEV)
    tables = c.tables.copy()
    tables[4, 4] = c.nb        # tokens 64 .. 79
    tables[6, 6] = -7          # tokens 96 .. 99
    _call(c, desc_of(kind, 4, 2, 64), new, q, out, tables=tables, most=most)
    got = out.cpu().numpy()
    at = np.cumsum([0] + new)
    assert (got[at[1]:at[2]] == 0).all() and np.isnan(got[at[2]:at[4]]).all()
    for b, first in ((4, 64), (6, 96)):
        rows, hidden = got[at[b]:at[b + 1]], first - (lens[b] - new[b])
        assert np.isnan(rows[hidden:]).all() and np.isfinite(rows[:hidden]).all()
        want, tol = reference(c, b, qv[at[b]:at[b + 1]])
        assert (np.abs(rows - want) <= tol)[:hidden].all()
    _check(c, new, out, qv, False, skip=(1, 2, 3, 4, 6))


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx4"])
def test_rising_scores(kind):
    """The row's maximum moves tile by tile, by more and by less than the reference's slack."""
    rng = np.random.default_rng(6)
    c = Cache(kind, 1, 64, [640], rng)
    q, qv = queries(kind, (640, 2, 64), rng)
    q[:] = 1.0
    qv[:] = 1.0
    x = np.repeat(np.cumsum(rng.uniform(0, 2.0, 640))[:, None], 64, 1) * 0.25
    from tests._cached import store
    blocks = np.zeros((c.nb, 1, BS, 64))
    blocks[c.tables[0, :40], 0] = x.reshape(40, BS, 64)
    c.k, c.ks = store(kind, blocks, False)
    out = torch.zeros((640, 2, 64), device=DEV)
    _call(c, desc_of(kind, 2, 1, 64), [640], q, out)
    _check(c, [640], out, qv, False)


def test_many_sequences():
    """More sequences than a wave searches in one step, most with one token or none."""
    rng = np.random.default_rng(7)
    new = rng.integers(0, 3, 4500)
    lens = np.maximum(new, rng.integers(0, 40, 4500))
    c = Cache("bf16", 1, 64, lens, rng)
    q, qv = queries("bf16", (int(new.sum()), 2, 64), rng)
    out = torch.zeros((int(new.sum()), 2, 64), device=DEV)
    _call(c, desc_of("bf16", 2, 1, 64), list(new), q, out)
    _check(c, list(new), out, qv, False)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_offsets_past_32_bits(kind):
    """The last blocks of a cache of over 4 GiB per tensor."""
    rng = np.random.default_rng(8)
    c = Cache(kind, 8, 128, [150, 33], rng, spare=0)
    k, v, ks, vs = c.device()
    per = k[0].numel()
    nb = (1 << 32) // (per * k.element_size()) + c.nb
    big = [torch.empty((nb, per), dtype=x.dtype, device=DEV) for x in (k, v)]
    for x, y in zip(big, (k, v)):
        x[nb - c.nb:] = y.reshape(c.nb, -1)
    sc = [None if s is None else torch.cat([torch.ones(nb - c.nb, device=DEV), s]) for s in (ks, vs)]
    t = np.where(c.tables >= 0, c.tables + (nb - c.nb), c.tables).astype(np.int32)
    q, qv = queries(kind, (60, 16, 128), rng)
    out = torch.zeros((60, 16, 128), device=DEV)
    _call(c, desc_of(kind, 16, 8, 128), [50, 10], q, out, tables=t, caches=(*big, *sc), nb=nb)
    _check(c, [50, 10], out, qv, False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,d", [(6, 2, 128), (9, 3, 64)])
def test_long_chunks(kind, hq, hkv, d):
    """Several row and token tiles to a sequence, chunk and length not multiples of either."""
    rng = np.random.default_rng(20)
    lens, new = [700, 333, 1030, 65], [650, 333, 514, 64]
    c = Cache(kind, hkv, d, lens, rng)
    c.poison()
    q, qv = queries(kind, (sum(new), hq, d), rng, 2.0)
    out = torch.zeros((sum(new), hq, d), device=DEV)
    _call(c, desc_of(kind, hq, hkv, d), new, q, out)
    _check(c, new, out, qv, False)


@pytest.mark.parametrize("hq,hkv,d", [(7, 1, 128), (2, 2, 64)])
def test_fp8_scales_of_any_sign(hq, hkv, d):
    """K and V scales that are zero, negative, tiny and large, one block or several to a tile."""
    rng = np.random.default_rng(21)
    lens, new = [200, 77], [150, 77]
    c = Cache("fp8", hkv, d, lens, rng)
    t = c.tables
    c.ks[t[0, 1]], c.ks[t[0, 6]] = 0.0, -c.ks[t[0, 6]]
    c.vs[t[0, 2]], c.vs[t[0, 5]], c.vs[t[0, 9]] = 0.0, -c.vs[t[0, 5]], 1e-30
    c.ks[t[1, 0]], c.vs[t[1, 0]], c.vs[t[1, 3]] = 1e-30, 0.0, 3.0
    q, qv = queries("fp8", (sum(new), hq, d), rng)
    out = torch.zeros((sum(new), hq, d), device=DEV)
    _call(c, desc_of("fp8", hq, hkv, d), new, q, out)
    _check(c, new, out, qv, False)


def test_two_streams():
    """Two calls at once, each with its own workspace and output, give what they give alone."""
    rng = np.random.default_rng(22)
    lens, new = [3000, 500, 40], [9, 200, 40]
    c = Cache("bf16", 2, 128, lens, rng)
    q, _ = queries("bf16", (sum(new), 8, 128), rng)
    desc, n, most = desc_of("bf16", 8, 2, 128), len(lens), 3000
    offs, t, dl = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), _up(c.tables), _up(c.lens)
    cache = c.device()
    size = tts_paged_prefill_workspace_size(desc, n, sum(new), most)
    ws = [torch.zeros(max(size, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    out = [torch.zeros((sum(new), 8, 128), device=DEV) for _ in range(3)]
    call = lambda i, s, o: tts_paged_prefill_attn(  # noqa: E731
        desc, n, sum(new), offs, q, *cache, t, t.shape[1], dl, most, c.nb, o, ws[i], size, s)
    call(0, None, out[2])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i, s in enumerate(streams):
            call(i, s, out[i])
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[2])
