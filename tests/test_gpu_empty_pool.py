"""Attention calls on a pool of no blocks: every id is outside it, so sequences with tokens have NaN rows and those without
zero rows."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import (tts_build_prefix_meta, tts_paged_decode_attn, tts_paged_decode_workspace_size,
                                  tts_paged_prefill_attn, tts_paged_prefill_workspace_size, tts_prefix_decode_attn,
                                  tts_prefix_decode_workspace_size)
from tests._cached import BS, DEV, KINDS, Cache, desc_of, queries

pytestmark = pytest.mark.gpu
LENS = [40, 0, 1]
NAN = np.array([True, False, True])


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _setup(kind, hq, hkv):
    c = Cache(kind, hkv, 64, LENS, np.random.default_rng(0), cols=64)
    q, _ = queries(kind, (3, hq, 64), np.random.default_rng(1))
    return c, desc_of(kind, hq, hkv, 64), q, torch.full((3, hq, 64), 5.0, device=DEV)


def _check(out):
    got = out.cpu().numpy()
    assert np.isnan(got[NAN]).all() and (got[~NAN] == 0).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(6, 2), (36, 2)])
@pytest.mark.parametrize("most", [40, 1024])
def test_paged(kind, hq, hkv, most):
    c, desc, q, out = _setup(kind, hq, hkv)
    size = tts_paged_decode_workspace_size(desc, 3, most)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    tts_paged_decode_attn(desc, 3, q, *c.device(), _up(c.tables), 64, _up(c.lens), most, 0, out, ws, size)
    _check(out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("most", [40, 1024])
def test_prefill(kind, most):
    c, desc, q, out = _setup(kind, 6, 2)
    size = tts_paged_prefill_workspace_size(desc, 3, 3, most)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    offs = _up(np.arange(4, dtype=np.int32))
    tts_paged_prefill_attn(desc, 3, 3, offs, q, *c.device(), _up(c.tables), 64, _up(c.lens), most, 0, out, ws, size)
    _check(out)


@pytest.mark.parametrize("kind", KINDS)
def test_prefix_beams_that_grew(kind):
    """Built for beams without tokens, which have some now."""
    c, desc, q, out = _setup(kind, 6, 2)
    meta = tts_build_prefix_meta(np.array([0, 3], np.int32), c.tables, np.zeros(3, np.int32), BS, 0, desc=desc)
    size = tts_prefix_decode_workspace_size(desc, meta)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    tts_prefix_decode_attn(desc, meta, q, *c.device(), _up(c.tables), 64, _up(c.lens), 0, out, ws, size)
    _check(out)
