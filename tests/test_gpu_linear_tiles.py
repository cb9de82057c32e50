"""Every kernel of the projections that a call can get, on rows apart: values, rows and gaps that stay as they are,
residuals in place, values that are not finite, repeats."""

import math

import pytest
import torch

from paper_2509_00195_amd import (make_linear, tts_gated_linear, tts_gated_linear_workspace_size, tts_linear,
                                  tts_linear_workspace_size)
from tests import _layer as L
from tests._linear_tiles import TILES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", list(TILES), ids=lambda t: "-".join(map(str, t)))
def test_kernel(kernel):
    kind, gated, _, _, _, aligned, split = kernel
    m, k, n = TILES[kernel]
    g = L.generator(m + k + n)
    gap, offset = (8, 0) if aligned else (3, 1)
    if aligned:  # (a row and its gap are whole pieces of 16 bytes)
        assert (k + gap) * (4 if kind == "f32" else 2) % 16 == 0
    x, w = L.rows((m, k), gap, kind, g, offset=offset), L.rows((n, k), gap, kind, g, k ** -0.5, offset=offset)
    u = L.rows((n, k), gap, kind, g, k ** -0.5, offset=offset) if gated else None
    bias = L.rows((1, n), 0, kind, g)[0]
    res = None if gated else L.rows((m, n), 0, kind, g)
    desc = make_linear(k, n, kind, kind, "silu")
    size = (tts_gated_linear_workspace_size if gated else tts_linear_workspace_size)(desc, m)
    assert size > 0 or not split
    ws = torch.full((size + 64,), 99, dtype=torch.uint8, device=L.DEV)
    flat = torch.full((offset + (m + 2) * (n + gap),), 7.0, dtype=L.TYPES[kind], device=L.DEV)
    out = flat[offset:].view(m + 2, n + gap)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:m, :n] = False

    def call():
        flat.fill_(7.0)
        y = out[:m, :n]
        if gated:
            tts_gated_linear(desc, m, x, w, u, y, bias, None, ws, size)
        else:
            y.copy_(res)
            tts_linear(desc, m, x, w, y, bias, y, ws, size)
        assert bool((out[rest] == 7.0).all()) and bool((flat[:offset] == 7.0).all()) and bool((ws[size:] == 99).all())
        return y.clone()

    y = call()
    L.close(y, *(L.gated(x, w, u, bias) if gated else L.linear(x, w, bias, "silu", res)), kind)
    assert torch.equal(call(), y)
    # Values that are not finite reach their row (of x) or their column (of weights) and nothing else.
    row, col = m // 2, n // 3
    x[row, k - 1], w[col, 0] = math.nan, math.inf
    z = call()
    keep = torch.ones((m, n), dtype=torch.bool, device=L.DEV)
    keep[row], keep[:, col] = False, False
    assert torch.equal(z[keep], y[keep]) and bool(torch.isnan(z[row]).all())
    keep.fill_(False)
    keep[:, col] = True
    keep[row] = False
    assert not bool(torch.isfinite(z[keep & (x[:, :1] > 0).expand(m, n)]).any())


def test_large_split_tiles_captured_and_replayed():
    """One workspace for all calls of a graph, one after the other; replays beside eager work of the same sizes."""
    kernels = [t for t in TILES if t[2] != 0 and t[6]]
    assert len(kernels) >= 10
    g = L.generator(2)
    calls, most = [], 0
    for t in kernels:
        kind, gated, aligned = t[0], t[1], t[5]
        m, k, n = TILES[t]
        gap = 8 if aligned else 3
        x, w, u = L.rows((m, k), gap, kind, g), *(L.rows((n, k), gap, kind, g, k ** -0.5) for _ in range(2))
        desc = make_linear(k, n, kind, kind, "relu")
        size = (tts_gated_linear_workspace_size if gated else tts_linear_workspace_size)(desc, m)
        most = max(most, size)
        calls.append((gated, desc, m, x, w, u, [torch.empty((m, n), dtype=L.TYPES[kind], device=L.DEV) for _ in range(2)]))
    ws = torch.empty(most, dtype=torch.uint8, device=L.DEV)

    def run(which, stream=None):
        for gated, desc, m, x, w, u, out in calls:
            if gated:
                tts_gated_linear(desc, m, x, w, u, out[which], None, None, ws, most, stream)
            else:
                tts_linear(desc, m, x, w, out[which], None, None, ws, most, stream)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        run(0, side)
    for rep in range(3):
        for c in calls:
            c[3].copy_(torch.randn(c[3].shape, generator=g, device=L.DEV))
        run(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, c in zip(kernels, calls):
            assert torch.equal(*c[6]), (rep, t)
