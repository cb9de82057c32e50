"""Random paged caches of every type for the tests of the operators around cached attention."""

from __future__ import annotations

import math

import numpy as np
import torch

from oracle.cached_ops import cache_values, chunk_attention, mx4_blocks, mx4_quantise
from paper_2509_00195_amd import make_desc

BS = 16
DEV = "cuda:0"
KINDS = ["f32", "bf16", "fp8", "mx4"]


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16)


def bits(x):
    return bf16(x).view(torch.int16).numpy().view(np.uint16)


def store(kind, x, values):
    """(storage, scales) of blocks of values x [nb][hkv][16][d]."""
    if kind == "mx4":
        return mx4_blocks(*mx4_quantise(x), values), None
    y = np.swapaxes(x, -1, -2) if values else x
    if kind == "f32":
        return np.ascontiguousarray(y, np.float32), None
    if kind == "bf16":
        return bits(y), None
    s = (np.abs(y).reshape(len(y), -1).max(1) / 448).astype(np.float32)
    t = torch.from_numpy(np.ascontiguousarray(y / s[:, None, None, None], np.float32)).clamp(-448, 448)
    return t.to(torch.float8_e4m3fn).view(torch.uint8).numpy(), s


class Cache:
    """Blocks of random values in storage form (host), a shuffled table per sequence."""

    def __init__(self, kind, hkv, d, lens, rng, spare=3, cols=None, gain=1.0):
        self.kind, self.hkv, self.d, self.lens = kind, hkv, d, np.asarray(lens, np.int32)
        need = [max(0, -(-int(n) // BS)) for n in self.lens]
        self.nb = sum(need) + spare
        cols = cols or max(need + [1]) + 1
        self.tables = np.full((len(need), cols), -1, np.int32)
        ids, at = rng.permutation(self.nb), 0
        for b, n in enumerate(need):
            self.tables[b, :n] = ids[at:at + n]
            at += n
        self.k, self.ks = store(kind, gain * rng.standard_normal((self.nb, hkv, BS, d)), False)
        self.v, self.vs = store(kind, rng.standard_normal((self.nb, hkv, BS, d)), True)

    def device(self):
        up = lambda a: None if a is None else torch.from_numpy(  # noqa: E731
            np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).to(DEV)
        return tuple(up(a) for a in (self.k, self.v, self.ks, self.vs))

    def dense(self, b, length=None):
        """float64 (k, v) [hkv][length][d] of sequence b."""
        n = int(self.lens[b]) if length is None else length
        ids = self.tables[b, :-(-n // BS)]
        pick = lambda c, s, values: np.swapaxes(cache_values(  # noqa: E731
            self.kind, c[ids], None if s is None else s[ids], self.d, values), 0, 1).reshape(self.hkv, -1, self.d)[:, :n]
        return pick(self.k, self.ks, False), pick(self.v, self.vs, True)

    def poison(self):
        """Unused slots of partly filled blocks and unused blocks hold NaN (types that have one)."""
        used = {}
        for b, n in enumerate(self.lens):
            for j in range(-(-int(n) // BS)):
                p = int(self.tables[b, j])
                used[p] = max(used.get(p, 0), min(BS, int(n) - j * BS))
        for p in range(self.nb):
            f = used.get(p, 0)
            if self.kind == "mx4":
                half = BS * self.d // 2
                ks = self.k[p][:, half:].reshape(self.hkv, BS, -1)
                vs = self.v[p][:, half:].reshape(self.hkv, -1, BS)
                ks[:, f:], vs[:, :, f:] = 255, 255
                continue
            nan = {"f32": np.nan, "bf16": 0x7FC0, "fp8": 0x7F}[self.kind]
            self.k[p, :, f:], self.v[p, :, :, f:] = nan, nan


def desc_of(kind, hq, hkv, d, out="f32"):
    return make_desc(hq, hkv, d, BS, "f32" if kind == "f32" else "bf16", kind, out)


def queries(kind, shape, rng, gain=1.0):
    """(device tensor, float64 values)."""
    x = gain * rng.standard_normal(shape)
    t = torch.from_numpy(x.astype(np.float32)) if kind == "f32" else bf16(x)
    return t.to(DEV), t.double().numpy()


def reference(cache, b, q, length=None):
    """(out, tolerance of an fp32 output) of the last len(q) tokens of sequence b; q float64 [n][hq][d].

    A probability is rounded to bf16 (2^-8 of itself at most), in the product and in the sum; a split's states to
    fp16 (2^-11); a score is off by its fp32 sum's roundings, (d + 8) 2^-24 of the sum of |q k|, and exp2 by 2^-20
    with its argument's (2^-24 of the score in log2 units, at most the same sum's); fp32 sums over the tokens by
    2^-24 each. All relative to the sum of p |v|. fp32 caches round no probability.
    A split's fp16 states share a power of two per row, which takes the row's largest element to [1/2, 1): an element
    below 2^-14 is off by up to half of fp16's smallest step there, 2^-25, which is 2^-24 of that largest element at
    most; over the splits, 2^-24 of the sum of p max |v|."""
    k, v = cache.dense(b, length)
    sc = 1.0 / math.sqrt(cache.d)
    out, bound, widest = chunk_attention(q, k, v, len(q), sc)
    g = q.shape[1] // cache.hkv
    most = max((np.abs(k[h // g]) @ np.abs(q[:, h]).T).max() for h in range(q.shape[1])) * sc
    rel = 2 * most * (cache.d + 10) * 2.0 ** -24 + 2.0 ** -20 + k.shape[1] * 2.0 ** -23
    if cache.kind != "f32":
        rel += 2 * 2.0 ** -8 + 2.0 ** -11
        return out, rel * bound + 2.0 ** -24 * widest
    return out, rel * bound + 1e-30


def close(got, want, tol, rounded=False):
    """`rounded`: the output is bf16, half a step (2^-8 of it) off what the kernel had."""
    got = got.double().cpu().numpy()
    err = np.abs(got - want)
    lim = tol + (2.0 ** -8 * (np.abs(want) + tol) if rounded else 0.0)
    assert np.isfinite(got).all()
    assert (err <= lim).all(), float((err / lim).max())
