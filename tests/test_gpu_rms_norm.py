"""The norm of hidden states against 64 bits."""

import math

import pytest
import torch

from paper_2509_00195_amd import make_norm, tts_rms_norm
from tests import _layer as L

pytestmark = pytest.mark.gpu


def run(x, weight, out, kind, out_kind, eps=1e-6, rows=None, stream=None):
    tts_rms_norm(make_norm(x.shape[1], eps, kind, out_kind), x.shape[0] if rows is None else rows, x, weight, out, stream)
    return out


@pytest.mark.parametrize("kind,out_kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("m,k", [(1, 1), (3, 7), (5, 8), (64, 1536), (7, 3584), (2, 8191), (2, 8192), (3, 8193), (2, 20001),
                                 (1, 70000), (3000, 40)])
def test_rows(kind, out_kind, m, k):
    g = L.generator(m + k)
    x = L.rows((m, k), 0, kind, g) * torch.exp(torch.randn((m, 1), generator=g, device=L.DEV)).to(L.TYPES[kind])
    w = L.rows((1, k), 0, kind, g)[0]
    for weight in (w, None):
        out = torch.full((m, k), math.nan, dtype=L.TYPES[out_kind], device=L.DEV)
        run(x, weight, out, kind, out_kind)
        L.close(out, *L.rms(x, weight, 1e-6), out_kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("k,gap,offset", [(200, 8, 0), (200, 3, 0), (200, 8, 1), (193, 0, 0), (8200, 5, 3)])
def test_rows_apart_and_in_place(kind, k, gap, offset):
    g = L.generator(gap)
    m = 9
    x = L.rows((m + 2, k), gap, kind, g, offset=offset)
    w = L.rows((1, k), 0, kind, g, offset=offset)[0]
    want = L.rms(x[:m], w, 1e-5)
    flat = torch.full((offset + (m + 2) * (k + gap),), 7.0, dtype=L.TYPES[kind], device=L.DEV)
    out = flat[offset:].view(m + 2, k + gap)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:m, :k] = False
    run(x, w, out[:, :k], kind, kind, 1e-5, rows=m)
    L.close(out[:m, :k], *want, kind)
    assert bool((out[rest] == 7.0).all()) and bool((flat[:offset] == 7.0).all())
    run(x, w, x, kind, kind, 1e-5, rows=m)
    assert torch.equal(x[:m], out[:m, :k])


def test_zeros_and_values_that_are_not_finite():
    x = torch.randn((5, 300), device=L.DEV)
    clean = run(x, None, torch.empty_like(x), "f32", "f32")
    y = x.clone()
    y[1, 7], y[2, 299], y[3] = math.inf, math.nan, 0.0
    out = run(y, None, torch.empty_like(x), "f32", "f32")
    assert torch.equal(out[[0, 4]], clean[[0, 4]])
    assert bool(torch.isnan(out[1, 7])) and bool((out[1, :7] == 0).all()) and bool(torch.isnan(out[2]).all())
    assert bool((out[3] == 0).all())
    assert bool(torch.isnan(run(y, None, torch.empty_like(x), "f32", "f32", 0.0)[3]).all())


def test_many_rows_and_offsets_past_32_bits():
    """More rows than workgroups of one launch, over 2^31 elements."""
    m, k = (1 << 20) + 33, 2064
    g = L.generator(4)
    x = torch.empty((m, k), dtype=torch.bfloat16, device=L.DEV)
    some = torch.tensor([0, 1, 1 << 19, (1 << 20) - 1, 1 << 20, m - 1], device=L.DEV)
    x.fill_(1.0)
    x[some] = L.rows((6, k), 0, "bf16", g)
    out = torch.empty_like(x)
    run(x, None, out, "bf16", "bf16")
    L.close(out[some], *L.rms(x[some], None, 1e-6), "bf16")
    assert bool((out[2] == 1).all()) and bool((out[m - 2] == 1).all())
