"""One workspace, made for the largest batch, serves the smaller ones."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import tts_paged_decode_attn, tts_paged_decode_workspace_size
from tests._cached import DEV, KINDS, Cache, close, desc_of, queries, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
def test_batches_that_shrink(kind):
    rng = np.random.default_rng(0)
    hq, hkv, d, most = 8, 4, 64, 1024
    c = Cache(kind, hkv, d, rng.integers(1, 700, 140), rng)
    desc = desc_of(kind, hq, hkv, d)
    size = tts_paged_decode_workspace_size(desc, 140, most)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    q, qv = queries(kind, (140, hq, d), rng)
    tables, lens, cache = torch.from_numpy(c.tables).to(DEV), torch.from_numpy(c.lens).to(DEV), c.device()
    pad = torch.full((140, most // 16), -1, dtype=torch.int32, device=DEV)
    pad[:, :tables.shape[1]] = tables[:, :most // 16]
    for n in (140, 128, 127, 60, 5, 1):
        out = torch.full((140, hq, d), 5.0, device=DEV)
        tts_paged_decode_attn(desc, n, q, *cache, pad, pad.shape[1], lens, most, c.nb, out, ws, size)
        assert (out[n:] == 5).all()
        for b in range(0, n, max(1, n // 5)):
            want, tol = reference(c, b, qv[b][None])
            close(out[b][None], want, tol)


def test_an_unsplit_batch_needs_no_workspace():
    """4-bit, 512 (sequence, KV head) pairs: no split, and NULL is taken."""
    rng = np.random.default_rng(1)
    c = Cache("mx4", 4, 64, rng.integers(1, 300, 128), rng)
    q, qv = queries("mx4", (128, 8, 64), rng)
    out = torch.zeros((128, 8, 64), device=DEV)
    tables = torch.from_numpy(c.tables).to(DEV)
    tts_paged_decode_attn(desc_of("mx4", 8, 4, 64), 128, q, *c.device(), tables, tables.shape[1],
                          torch.from_numpy(c.lens).to(DEV), 300, c.nb, out, None, 0)
    for b in (0, 77, 127):
        want, tol = reference(c, b, qv[b][None])
        close(out[b][None], want, tol)
