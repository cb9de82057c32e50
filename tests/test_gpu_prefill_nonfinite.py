"""Values that are not finite at tokens that prefill queries see: what the formula makes of them, in whatever tile the query
stands."""

import math

import numpy as np
import pytest
import torch

from oracle.cached_ops import chunk_attention
from paper_2509_00195_amd import tts_paged_prefill_attn, tts_paged_prefill_workspace_size
from tests._cached import BS, DEV, Cache, desc_of, queries, reference

pytestmark = pytest.mark.gpu


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _call(c, hq, new, q):
    desc, total = desc_of(c.kind, hq, c.hkv, c.d), int(q.shape[0])
    most = int(c.lens.max())
    size = tts_paged_prefill_workspace_size(desc, len(c.lens), total, most)
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, 5.0, device=DEV)
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tts_paged_prefill_attn(desc, len(c.lens), total, _up(offs), q, *c.device(), _up(c.tables), c.tables.shape[1], _up(c.lens),
                           most, c.nb, out, ws, size)
    return out.cpu().numpy(), size > 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,length,split", [(40, 400, False), (1, 400, None), (1, 2600, True)])
def test_visible_infinities(kind, d, seqs, length, split):
    """+inf, -inf and both in dims of one head's values; queries whose tile holds hidden tokens and queries past it."""
    n, first = 200, length - 200
    make = lambda: Cache(kind, 2, d, [length] * seqs, np.random.default_rng(0))  # noqa: E731
    c, clean = make(), make()
    pos, neg, nan = (np.inf, -np.inf, np.nan) if kind == "f32" else (0x7F80, 0xFF80, 0x7FC0)
    for token, dim, x in ((first + 5, 3, pos), (first + 70, 7, neg), (first + 71, 40, pos), (first + 130, 40, neg),
                          (20, 50, neg), (first + 64, 51, nan), (first + 199, 52, pos)):
        c.v[c.tables[0, token // BS], 1, dim, token % BS] = x
    q, qv = queries(kind, (n * seqs, 6, d), np.random.default_rng(1))
    got, used = _call(c, 6, [n] * seqs, q)
    assert split is None or used == split
    assert np.isfinite(got[n:]).all()
    got, qv = got[:n], qv[:n]
    k, v = c.dense(0)
    with np.errstate(invalid="ignore"):
        want = chunk_attention(qv, k, v, n, 1.0 / math.sqrt(d))[0]
    _, tol = reference(clean, 0, qv)
    assert np.isposinf(want).any() and np.isneginf(want).any() and np.isnan(want).any()
    for f in (np.isposinf, np.isneginf, np.isnan):
        assert (f(got) == f(want)).all()
    keep = np.isfinite(want)
    assert (np.abs(got - np.where(keep, want, 0)) <= tol)[keep].all()


@pytest.mark.parametrize("scale", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("length", [100, 2600])
def test_fp8_scales_that_are_not_finite(scale, which, length):
    """The rows that see the block are NaN, the others as ever."""
    n, block = 100, length // BS - 2
    c = Cache("fp8", 1, 128, [length], np.random.default_rng(2))
    q, qv = queries("fp8", (n, 4, 128), np.random.default_rng(3))
    want, tol = reference(c, 0, qv)
    (c.ks if which == "k" else c.vs)[c.tables[0, block]] = scale
    got, _ = _call(c, 4, [n], q)
    first = block * BS - (length - n)
    assert np.isnan(got[first:]).all()
    assert (np.abs(got - want) <= tol)[:first].all()
