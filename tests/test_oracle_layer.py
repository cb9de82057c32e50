"""Pins of the plain forms that the layer's operators are compared with (CPU)."""

import math

import numpy as np
import pytest
import torch

from oracle.layer_ops import head_norm
from tests import _layer as L


def test_head_norm():
    x = np.array([[3.0, -4.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0]], np.float32)
    y = head_norm(x, None, 0.0)
    assert np.array_equal(y[0], np.array([1.2, -1.6, 0, 0], np.float32)) and np.isnan(y[1]).all()
    assert np.array_equal(head_norm(x, None, 1.0)[1], np.zeros(4, np.float32))
    w = np.array([2.0, 0.5, 1.0, -1.0], np.float32)
    assert np.array_equal(head_norm(x, w, 0.0)[0], y[0] * w)
    rng = np.random.default_rng(0)
    z = rng.standard_normal((5, 64)).astype(np.float32)
    n = head_norm(z, None, 0.0).astype(np.float64)
    # root and two products of half a step each, on a mean of squares of 1
    assert np.abs((n * n).mean(-1) - 1).max() <= 4 * 2.0 ** -24


def test_activations():
    y = torch.tensor([-2.0, -0.5, 0.0, 1.0, 3.0], dtype=torch.float64)
    want = {
        "none": lambda v: v, "relu": lambda v: max(v, 0.0), "silu": lambda v: v / (1 + math.exp(-v)),
        "gelu": lambda v: v * 0.5 * (1 + math.erf(v / math.sqrt(2))),
        "gelu_tanh": lambda v: v * 0.5 * (1 + math.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))),
    }
    for act, f in want.items():
        assert torch.allclose(L.activate(y, act), torch.tensor([f(float(v)) for v in y], dtype=torch.float64), rtol=0, atol=1e-15)


@pytest.mark.parametrize("act", L.ACTS)
def test_no_activation_is_steeper_than_the_tolerance_has_it(act):
    y = torch.linspace(-12, 12, 200001, dtype=torch.float64)
    v = L.activate(y, act)
    assert ((v[1:] - v[:-1]).abs() / (y[1:] - y[:-1])).max() <= 1.13


def test_products_by_loops():
    rng = np.random.default_rng(1)
    x, w, u = (torch.from_numpy(rng.standard_normal(s)) for s in ((3, 5), (4, 5), (4, 5)))
    b, r = torch.from_numpy(rng.standard_normal(4)), torch.from_numpy(rng.standard_normal((3, 4)))
    out, _ = L.linear(x, w, b, "relu", r)
    both, _ = L.gated(x, w, u, b, None, "relu")
    for m in range(3):
        for n in range(4):
            g = sum(float(x[m, k]) * float(w[n, k]) for k in range(5)) + float(b[n])
            v = sum(float(x[m, k]) * float(u[n, k]) for k in range(5))
            assert abs(float(out[m, n]) - (max(g, 0.0) + float(r[m, n]))) < 1e-12
            assert abs(float(both[m, n]) - max(g, 0.0) * v) < 1e-12


def test_rms():
    x = torch.tensor([[3.0, 4.0], [0.0, 0.0]], dtype=torch.float64)
    out, _ = L.rms(x, torch.tensor([1.0, 2.0]), 0.5)
    s = math.sqrt(13.0)
    assert torch.allclose(out, torch.tensor([[3 / s, 8 / s], [0, 0]], dtype=torch.float64), rtol=1e-15, atol=0)
