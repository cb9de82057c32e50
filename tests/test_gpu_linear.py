"""Projections and the gated product against 64 bits."""

import math

import pytest
import torch

from paper_2509_00195_amd import (make_linear, tts_gated_linear, tts_gated_linear_workspace_size, tts_linear,
                                  tts_linear_workspace_size)
from tests import _layer as L

pytestmark = pytest.mark.gpu


def run_linear(x, w, out, kind, out_kind, act="none", bias=None, residual=None, n=None, stream=None):
    m = x.shape[0] if n is None else n
    desc = make_linear(x.shape[1], w.shape[0], kind, out_kind, act)
    size = tts_linear_workspace_size(desc, m)
    ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=L.DEV)
    tts_linear(desc, m, x, w, out, bias, residual, ws, size, stream)
    return out, ws


def run_gated(x, wg, wu, out, kind, out_kind, act="silu", bg=None, bu=None, stream=None):
    desc = make_linear(x.shape[1], wg.shape[0], kind, out_kind, act)
    size = tts_gated_linear_workspace_size(desc, x.shape[0])
    ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=L.DEV)
    tts_gated_linear(desc, x.shape[0], x, wg, wu, out, bg, bu, ws, size, stream)
    return out, ws


# Both kernels, each number of row tiles, whole and partial tiles and chunks, split and unsplit inner dimensions, the
# large tiles (the last one).
SHAPES = [(1, 1, 1), (1, 64, 16), (1, 2048, 2056), (3, 7, 5), (16, 128, 48), (17, 200, 100), (31, 1000, 2080), (32, 96, 30),
          (33, 1001, 333), (64, 640, 96), (64, 4096, 32), (65, 72, 130), (77, 3000, 20), (128, 128, 128), (129, 1000, 257),
          (200, 64, 64), (257, 8, 300), (300, 5120, 264), (513, 136, 40), (4101, 200, 4120)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear_shapes(kind, m, k, n):
    g = L.generator(m * 7 + k + n)
    x, w = L.rows((m, k), 0, kind, g), L.rows((n, k), 0, kind, g, k ** -0.5)
    bias = L.rows((1, n), 0, kind, g)[0]
    res = L.rows((m, n), 0, kind, g)
    out = torch.full((m, n), math.nan, dtype=L.TYPES[kind], device=L.DEV)
    run_linear(x, w, out, kind, kind, "silu", bias, res)
    L.close(out, *L.linear(x, w, bias, "silu", res), kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_gated_shapes(kind, m, k, n):
    g = L.generator(m * 5 + k + n)
    x = L.rows((m, k), 0, kind, g)
    wg, wu = (L.rows((n, k), 0, kind, g, k ** -0.5) for _ in range(2))
    out = torch.full((m, n), math.nan, dtype=L.TYPES[kind], device=L.DEV)
    run_gated(x, wg, wu, out, kind, kind)
    L.close(out, *L.gated(x, wg, wu), kind)


# Shapes that the plan gives to each of its tiles in turn, aligned rows (whole and partial tiles, several rounds of their
# stages) and others.
PLAIN_TILES = [(1, 624, 16), (1, 608, 4217), (1, 616, 8269), (1, 72, 26688), (17, 624, 2380), (17, 648, 4538),
               (17, 656, 8545), (35, 680, 6179), (36, 624, 6232), (101, 608, 6734), (931, 608, 8414), (322, 632, 10998),
               (131, 608, 11194), (67, 656, 9625), (200, 2048, 2056), (1, 607, 16), (1, 673, 9370), (1, 630, 8300), (17, 957, 8180),
               (17, 714, 2081), (18, 633, 4364), (19, 651, 8214), (33, 789, 6271), (35, 718, 6148), (39, 627, 11528),
               (534, 671, 170)]
GATED_TILES = [(1, 608, 16), (1, 608, 8288), (17, 720, 2155), (17, 624, 4365), (38, 608, 2698), (35, 624, 6956),
               (282, 640, 10897), (140, 608, 11253), (65, 616, 8802), (33, 712, 8240), (200, 2048, 1100), (1, 603, 16), (1, 625, 8272),
               (18, 615, 2274), (33, 618, 2806), (35, 766, 2724), (36, 633, 5530), (519, 638, 160)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", PLAIN_TILES)
def test_every_plain_tile(kind, m, k, n):
    g = L.generator(m + k)
    x, w = L.rows((m, k), 0, kind, g), L.rows((n, k), 0, kind, g, k ** -0.5)
    res = L.rows((m, n), 0, kind, g)
    out = torch.full((m, n), math.nan, dtype=L.TYPES[kind], device=L.DEV)
    run_linear(x, w, out, kind, kind, "none", None, res)
    L.close(out, *L.linear(x, w, None, "none", res), kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", GATED_TILES)
def test_every_gated_tile(kind, m, k, n):
    g = L.generator(m + k)
    x = L.rows((m, k), 0, kind, g)
    wg, wu = (L.rows((n, k), 0, kind, g, k ** -0.5) for _ in range(2))
    bg = L.rows((1, n), 0, kind, g)[0]
    out = torch.full((m, n), math.nan, dtype=L.TYPES[kind], device=L.DEV)
    run_gated(x, wg, wu, out, kind, kind, "gelu_tanh", bg)
    L.close(out, *L.gated(x, wg, wu, bg, None, "gelu_tanh"), kind)


@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("kind,out_kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("m", [5, 100])
def test_types_and_activations(kind, out_kind, act, m):
    g = L.generator(11)
    k, n = 168, 76
    x = L.rows((m, k), 0, kind, g, 3.0)
    w, u = (L.rows((n, k), 0, kind, g, k ** -0.5) for _ in range(2))
    b0, b1 = (L.rows((1, n), 0, kind, g)[0] for _ in range(2))
    res = L.rows((m, n), 0, out_kind, g)
    for bias, r in ((None, None), (b0, None), (None, res), (b0, res)):
        out = torch.empty((m, n), dtype=L.TYPES[out_kind], device=L.DEV)
        run_linear(x, w, out, kind, out_kind, act, bias, r)
        L.close(out, *L.linear(x, w, bias, act, r), out_kind)
    for bg, bu in ((None, None), (b0, None), (None, b1), (b0, b1)):
        out = torch.empty((m, n), dtype=L.TYPES[out_kind], device=L.DEV)
        run_gated(x, w, u, out, kind, out_kind, act, bg, bu)
        L.close(out, *L.gated(x, w, u, bg, bu, act), out_kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 40, 140])
@pytest.mark.parametrize("k,gap,offset", [(200, 8, 0), (200, 24, 8), (200, 3, 0), (200, 8, 1), (193, 0, 0), (193, 15, 3)])
def test_rows_apart(kind, m, k, gap, offset):
    """Gaps hold NaN, and rows begin at any element; gaps of the output, and what lies behind it, stay as they are."""
    g = L.generator(gap + offset)
    n = 90
    x, w = L.rows((m, k), gap, kind, g, offset=offset), L.rows((n, k), gap, kind, g, k ** -0.5, offset=offset)
    u = L.rows((n, k), gap, kind, g, k ** -0.5, offset=offset)
    res = L.rows((m, n), gap, kind, g, offset=offset)
    flat = torch.full((offset + (m + 2) * (n + gap),), 7.0, dtype=L.TYPES[kind], device=L.DEV)
    out = flat[offset:].view(m + 2, n + gap)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:m, :n] = False
    run_linear(x, w, out[:m, :n], kind, kind, "none", None, res)
    L.close(out[:m, :n], *L.linear(x, w, None, "none", res), kind)
    assert bool((out[rest] == 7.0).all()) and bool((flat[:offset] == 7.0).all())
    flat.fill_(7.0)
    run_gated(x, w, u, out[:m, :n], kind, kind)
    L.close(out[:m, :n], *L.gated(x, w, u), kind)
    assert bool((out[rest] == 7.0).all()) and bool((flat[:offset] == 7.0).all())


@pytest.mark.parametrize("m,k", [(20, 96), (20, 4096), (150, 96), (150, 4096)])
def test_rows_behind_the_last_and_the_workspace_behind_its_end(m, k):
    """Tensors of more rows than the call's: the others are neither read nor written; nor is more of the workspace."""
    g = L.generator(3)
    n = 64
    x, w = L.rows((m + 5, k), 0, "bf16", g), L.rows((n, k), 0, "bf16", g, k ** -0.5)
    x[m:] = math.nan
    out = torch.full((m + 5, n), 7.0, dtype=torch.bfloat16, device=L.DEV)
    desc = make_linear(k, n)
    size = tts_linear_workspace_size(desc, m)
    assert (size > 0) == (k == 4096)
    ws = torch.full((size + 4096,), 99, dtype=torch.uint8, device=L.DEV)
    tts_linear(desc, m, x, w, out, None, None, ws, size)
    L.close(out[:m], *L.linear(x[:m], w), "bf16")
    assert bool((out[m:] == 7.0).all()) and bool((ws[size:] == 99).all())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,k", [(9, 200), (9, 4096), (100, 200), (100, 4096), (100, 4095), (600, 96)])
def test_values_that_are_not_finite(kind, m, k):
    """They reach their row (of x) or their column (of weights) and nothing else; infinities add up as the formula has
    it."""
    g = L.generator(5)
    n = 80
    x, w = L.rows((m, k), 0, kind, g), L.rows((n, k), 0, kind, g, k ** -0.5)
    clean = torch.empty((m, n), dtype=L.TYPES[kind], device=L.DEV)
    run_linear(x, w, clean, kind, kind)
    x[3, 7], x[5, k - 1], w[11, k // 2] = math.nan, math.inf, -math.inf
    out = torch.empty_like(clean)
    run_linear(x, w, out, kind, kind)
    assert bool(torch.isnan(out[3]).all())
    ok = torch.ones(m, dtype=torch.bool, device=L.DEV)
    ok[[3, 5]] = False
    cols = torch.ones(n, dtype=torch.bool, device=L.DEV)
    cols[11] = False
    assert torch.equal(out[ok][:, cols], clean[ok][:, cols])
    assert torch.equal(out[5][cols], torch.where(w[cols, k - 1] > 0, math.inf, -math.inf).to(out.dtype))
    assert torch.equal(out[ok][:, 11], torch.where(x[ok, k // 2] > 0, -math.inf, math.inf).to(out.dtype))


@pytest.mark.parametrize("m,k", [(4, 512), (64, 4096), (90, 4096), (300, 100)])
@pytest.mark.parametrize("kind,out_kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_in_place_residual_and_repeats(m, k, kind, out_kind):
    g = L.generator(6)
    n = 200
    x, w = L.rows((m, k), 0, kind, g), L.rows((n, k), 0, kind, g, k ** -0.5)
    res = L.rows((m, n), 0, out_kind, g)
    apart = torch.empty_like(res)
    run_linear(x, w, apart, kind, out_kind, "gelu", None, res)
    for _ in range(3):
        same = res.clone()
        run_linear(x, w, same, kind, out_kind, "gelu", None, same)
        assert torch.equal(same, apart)


def test_halves_of_one_weight():
    """Gate and up as the halves of one tensor, and as every other row of one."""
    g = L.generator(8)
    m, k, n = 70, 264, 150
    x, both = L.rows((m, k), 0, "bf16", g), L.rows((2 * n, k), 0, "bf16", g, k ** -0.5)
    for wg, wu in ((both[:n], both[n:]), (both[0::2], both[1::2])):
        out = torch.empty((m, n), dtype=torch.bfloat16, device=L.DEV)
        run_gated(x, wg, wu, out, "bf16", "bf16")
        L.close(out, *L.gated(x, wg, wu), "bf16")


@pytest.mark.parametrize("m", [1, 64, 65, 320])
def test_a_smaller_call_in_a_larger_ones_workspace(m):
    g = L.generator(9)
    k, n = 8192, 144
    desc = make_linear(k, n)
    size = tts_linear_workspace_size(desc, 320)
    ws = torch.empty(size, dtype=torch.uint8, device=L.DEV)
    x, w = L.rows((m, k), 0, "bf16", g), L.rows((n, k), 0, "bf16", g, k ** -0.5)
    out = torch.empty((m, n), dtype=torch.bfloat16, device=L.DEV)
    tts_linear(desc, m, x, w, out, None, None, ws, size)
    L.close(out, *L.linear(x, w), "bf16")


def test_offsets_that_pass_32_bits():
    """Weights and an output of more than 2^31 elements, the last columns' own."""
    g = L.generator(10)
    k, n = 64, (1 << 25) + 40
    x = L.rows((70, k), 0, "bf16", g)
    w = torch.zeros((n, k), dtype=torch.bfloat16, device=L.DEV)
    w[-100:] = L.rows((100, k), 0, "bf16", g, 0.125)
    out = torch.full((70, n), math.nan, dtype=torch.bfloat16, device=L.DEV)
    for m in (3, 70):
        out.fill_(math.nan)
        run_linear(x[:m], w, out[:m], "bf16", "bf16")
        L.close(out[:m, -100:], *L.linear(x[:m], w[-100:]), "bf16")
        assert bool((out[:m, :-100] == 0).all())


def test_captured_and_replayed():
    """Split and unsplit calls in one graph, sharing a workspace one after the other: every replay leaves what the eager
    calls leave."""
    g = L.generator(12)
    shapes = [(7, 4096, 96), (64, 512, 1200), (90, 4096, 100), (300, 264, 140)]
    cases = []
    for m, k, n in shapes:
        x, w, u = L.rows((m, k), 0, "bf16", g), *(L.rows((n, k), 0, "bf16", g, k ** -0.5) for _ in range(2))
        d, size = make_linear(k, n, act="silu"), 0
        size = max(tts_linear_workspace_size(d, m), tts_gated_linear_workspace_size(d, m))
        outs = [torch.empty((m, n), dtype=torch.bfloat16, device=L.DEV) for _ in range(4)]
        cases.append((d, m, x, w, u, outs, size))
    most = max(c[-1] for c in cases)
    ws = torch.empty(most, dtype=torch.uint8, device=L.DEV)

    def step(first, stream=None):
        for d, m, x, w, u, outs, _ in cases:
            tts_linear(d, m, x, w, outs[first], None, None, ws, most, stream)
            tts_gated_linear(d, m, x, w, u, outs[first + 1], None, None, ws, most, stream)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(0, side)
    for rep in range(4):
        for c in cases:
            c[2].copy_(torch.randn(c[2].shape, generator=g, device=L.DEV))
        step(2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for c in cases:
            assert torch.equal(c[5][0], c[5][2]) and torch.equal(c[5][1], c[5][3]), rep


def test_two_streams():
    g = L.generator(13)
    k, n = 4096, 100
    w = L.rows((n, k), 0, "bf16", g, k ** -0.5)
    xs = [L.rows((m, k), 0, "bf16", g) for m in (8, 90)]
    want = [run_linear(x, w, torch.empty((len(x), n), dtype=torch.bfloat16, device=L.DEV), "bf16", "bf16")[0] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [[torch.empty((len(x), n), dtype=torch.bfloat16, device=L.DEV) for _ in range(5)] for x in xs]
    desc = make_linear(k, n)
    size = [tts_linear_workspace_size(desc, len(x)) for x in xs]
    wss = [torch.empty(s, dtype=torch.uint8, device=L.DEV) for s in size]
    torch.cuda.synchronize()
    for i in range(5):
        for x, s, o, sz, ws in zip(xs, streams, outs, size, wss):
            tts_linear(desc, len(x), x, w, o[i], None, None, ws, sz, s)
    torch.cuda.synchronize()
    for o, v in zip(outs, want):
        assert all(torch.equal(y, v) for y in o)


# Shapes for each large tile whose columns are whole quads, where biases and residuals are loaded as quads: tiles that
# end in the middle, rows and columns.
QUADS = [(931, 608, 8416), (322, 632, 11000), (131, 608, 11196), (67, 656, 9624), (4101, 200, 4120), (534, 671, 172),
         (64, 4096, 36), (33, 712, 4)]


@pytest.mark.parametrize("kind,out_kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("m,k,n", QUADS)
def test_biases_and_residuals_as_quads(kind, out_kind, m, k, n):
    g = L.generator(m + n)
    x = L.rows((m, k), 0, kind, g)
    w, u = (L.rows((n, k), 0, kind, g, k ** -0.5) for _ in range(2))
    b0, b1 = (L.rows((1, n), 0, kind, g)[0] for _ in range(2))
    res = L.rows((m, n), 5, out_kind, g)
    for act in ("none", "gelu"):
        out = torch.full((m, n), math.nan, dtype=L.TYPES[out_kind], device=L.DEV)
        run_linear(x, w, out, kind, out_kind, act, b0, res)
        L.close(out, *L.linear(x, w, b0, act, res), out_kind)
    out = torch.full((m, n), math.nan, dtype=L.TYPES[out_kind], device=L.DEV)
    run_gated(x, w, u, out, kind, out_kind, "relu", b0, b1)
    L.close(out, *L.gated(x, w, u, b0, b1, "relu"), out_kind)
