"""Plain forms, in 64 bits, of the operators around a layer's cached attention, with how far a kernel may be off."""

from __future__ import annotations

import math

import numpy as np
import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]



def activate(y, act):
    if act == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == "silu":
        return y / (1 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * torch.erfc(-y / math.sqrt(2))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def act_tolerance(y, dy, act):
    """What an error dy of the argument and the function's own roundings make of the result. No activation is steeper
    than 1.13. SiLU and the tanh form take an exponential (2^-22 of itself, and its argument's, |y| or
    2 |z| < 4 |y| + |y|^3 roundings of 2^-24 each, which is what the sigmoid is off by relatively), a sum and a quotient
    (2^-22 together with the last product); GELU's erfc is good to 2^-20, its argument's two roundings change it by
    2 |y / sqrt 2| |y| 2^-23 relatively at most (the logarithmic slope of erfc grows as 2 x)."""
    if act in ("none", "relu"):
        return dy
    a = y.abs()
    steep = {"silu": a, "gelu_tanh": 4 * a + a ** 3, "gelu": a * a}[act]
    return 1.13 * dy + activate(y, act).abs() * (2.0 ** -20 + steep * 2.0 ** -23) + 1e-37


def product(x, w, bias):
    """Sums in 64 bits, and how far one in 32 bits may be off: each of its k additions, and the additions that join
    its parts, round a partial sum by 2^-24 at most; 2^-23 allows a matrix instruction that truncates inside."""
    x, w = x.double(), w.double()
    y = x @ w.t().contiguous()
    size = x.abs() @ w.abs().t().contiguous()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, size * (x.shape[1] + 40) * 2.0 ** -23 + 1e-37


def linear(x, w, bias=None, act="none", residual=None):
    y, dy = product(x, w, bias)
    out, tol = activate(y, act), act_tolerance(y, dy, act)
    if residual is not None:
        out = out + residual.double()
        tol = tol + out.abs() * 2.0 ** -24
    return out, tol


def gated(x, wg, wu, bg=None, bu=None, act="silu"):
    g, dg = product(x, wg, bg)
    u, du = product(x, wu, bu)
    a, da = activate(g, act), act_tolerance(g, dg, act)
    out = a * u
    return out, da * u.abs() + a.abs() * du + da * du + out.abs() * 2.0 ** -24


def close(got, want, tol, out_type):
    """The result is rounded once to its type."""
    err = (got.double() - want).abs()
    lim = tol + HALF_STEP[out_type] * (want.abs() + tol)
    assert torch.isfinite(got).all()
    assert bool((err <= lim).all()), float((err / lim).max())


def rows(shape, gap, kind, gen, scale=1.0, offset=0, fill=math.nan):
    """A tensor [rows][cols] of random values, `gap` elements of `fill` behind each row, `offset` elements into its
    storage."""
    n, cols = shape
    t = TYPES[kind]
    flat = torch.full((offset + n * (cols + gap) + 8,), fill, dtype=t, device=DEV)
    x = flat[offset:offset + n * (cols + gap)].view(n, cols + gap)[:, :cols]
    x.copy_((scale * torch.randn((n, cols), generator=gen, device=DEV)).to(t))
    return x


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rms(x, weight, eps):
    """(values, tolerance): a sum of squares in 32 bits is off by len 2^-24 of itself at most, half of which reaches the
    scale; root, quotient and products round a few times."""
    y = x.double()
    out = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps)))
    if weight is not None:
        out = out * weight.double()
    return out, out.abs() * (x.shape[-1] / 2 + 8) * 2.0 ** -24 + 1e-37
