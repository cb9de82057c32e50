"""The norm of hidden states at the ends of its ranges."""

import math

import pytest
import torch

from paper_2509_00195_amd import make_norm, tts_rms_norm
from tests import _layer as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [(1 << 31) - 8, (1 << 31) - 7, (1 << 31) - 1])
def test_the_longest_rows(k):
    """Every row length that an int32 holds. The squares are ones, and a thread adds at most 2^23 of them, so that its
    sum is exact; the 256 threads' add up to 2^31 - 8 or 2^31, at most 2^-24 of itself off."""
    x = torch.ones((1, k), dtype=torch.bfloat16, device=L.DEV)
    x[0, k // 3::7] = -1.0
    out = torch.full((1, k), math.nan, dtype=torch.bfloat16, device=L.DEV)
    tts_rms_norm(make_norm(k, 0.0), 1, x, None, out)
    assert torch.equal(out.view(torch.int16), x.view(torch.int16))  # 1 to within 2^-23, which bf16 rounds to 1


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-37, 2.0 ** -120])
@pytest.mark.parametrize("kind,out_kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("k", [8, 1000, 2048, 3584, 4096, 5001, 8200])
def test_an_eps_that_leaves_small_rows_their_own_scale(eps, kind, out_kind, k):
    """Rows whose squares vanish in fp32, rows whose squares pass it where eps is small enough for 64 bits, and rows of
    one element that is not zero. The tolerance is that of sums in 32 bits."""
    g = L.generator(k)
    sizes = [1.0, 1e-10, 1e-17, 1e-20, 1e-25, 1e-31, 1e-38] + ([1e20, 1e30, 1e37] if eps < 2.0 ** -120 else [])
    x = torch.randn((len(sizes) + 1, k), generator=g, device=L.DEV) * torch.tensor(sizes + [0.0], device=L.DEV)[:, None]
    x[-1, k // 2] = 1e-30
    x = x.to(L.TYPES[kind])
    w = L.rows((1, k), 0, kind, g)[0]
    for weight in (w, None):
        out = torch.full(x.shape, math.nan, dtype=L.TYPES[out_kind], device=L.DEV)
        tts_rms_norm(make_norm(k, eps, kind, out_kind), len(x), x, weight, out)
        L.close(out, *L.rms(x, weight, eps), out_kind)
        if kind == out_kind:
            same = x.clone()
            tts_rms_norm(make_norm(k, eps, kind, kind), len(x), same, weight, same)
            assert torch.equal(same, out)


@pytest.mark.parametrize("k", [300, 2048, 5001])
def test_values_that_are_not_finite_beside_an_eps_of_zero(k):
    x = torch.randn((6, k), device=L.DEV)
    y = x.clone()
    y[1, 7], y[2, k - 1], y[3], y[4] = math.inf, math.nan, 0.0, 1e-42
    out = torch.empty_like(y)
    tts_rms_norm(make_norm(k, 0.0, "f32", "f32"), 6, y, None, out)
    ok = torch.tensor([0, 5], device=L.DEV)
    L.close(out[ok], *L.rms(x[ok], None, 0.0), "f32")
    assert bool(torch.isnan(out[1, 7])) and bool((out[1, 8:] == 0).all()) and bool(torch.isnan(out[2]).all())
    assert bool(torch.isnan(out[3]).all()) and bool((out[4] == 1).all())
