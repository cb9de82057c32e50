"""Oracle of the operators around cached attention (test infrastructure).

Plain NumPy, written from the definitions:

* OCP Microscaling FP4: E2M1 codes (sign, two exponent bits of bias 1, one
  mantissa bit) under one E8M0 scale byte (value 2^(byte - 127), 255: NaN)
  per 32 head dims of a token; ``mx4_quantise`` finds each nearest code by
  search over the table of values, ties to the even code.
* the paged caches' storage: ``cache_values`` gives the values of whole
  blocks of any cache type, ``mx4_blocks`` / ``mx4_unblocks`` the 4-bit
  storage (codes, then scales).
* ``rope``: the rotation of a head's pairs, in fp32, each product and the sum
  rounded; in fp64 with ``exact=True``.
* ``append_chunk``: new tokens of one sequence into its blocks (fp8: the
  block's scale set or raised once for all of them).
* ``chunk_attention``: causal attention of a sequence's last tokens over
  gathered keys and values in fp64, with the sum of p |v| that bounds what
  rounding the probabilities can change, and the sum of p max |v| (the
  largest over the dims), which bounds what a row of common scale can.
"""

from __future__ import annotations

import numpy as np

from .fp8 import e4m3_table
from .kv_ops import e4m3_encode

GROUP = 32
BLOCK = 16
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_value(code: int) -> float:
    """From the bit formula: s eem; e = 0 is m / 2, else 2^(e - 1) (1 + m / 2)."""
    s, e, m = code >> 3 & 1, code >> 1 & 3, code & 1
    v = m / 2.0 if e == 0 else 2.0 ** (e - 1) * (1.0 + m / 2.0)
    return -v if s else v


def e8m0_value(byte) -> np.ndarray:
    b = np.asarray(byte).astype(np.int64)
    return np.where(b == 255, np.nan, np.exp2(b.astype(np.float64) - 127.0))


def mx4_quantise(x):
    """(codes uint8 [..., d], scale bytes uint8 [..., d / 32]) of float32 values."""
    x = np.asarray(x, np.float32)
    g = x.astype(np.float64).reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(divide="ignore", invalid="ignore"):
        top = np.max(np.abs(g), -1)
        e = np.floor(np.log2(top)) - 2 + 127
    finite = np.isfinite(g).all(-1)
    byte = np.where(finite, np.clip(np.where(np.isfinite(e), e, 1), 1, 254), 255).astype(np.int64)
    m = np.where(finite[..., None], g, 0.0) / np.exp2(np.where(finite, byte, 127).astype(np.float64) - 127.0)[..., None]
    a = np.abs(m)
    dist = np.abs(a[..., None] - E2M1)
    best = dist.min(-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = np.where(finite[..., None], code + 8 * np.signbit(m), 0)
    return code.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8)


def _pack(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def _unpack(b):
    out = np.empty((*b.shape[:-1], 2 * b.shape[-1]), np.uint8)
    out[..., 0::2], out[..., 1::2] = b & 15, b >> 4
    return out


def mx4_blocks(codes, scale, values):
    """Storage [..., 17 d / 2] of blocks from codes [..., 16, d] and scales [..., 16, d / 32]."""
    if values:
        codes, scale = np.swapaxes(codes, -1, -2), np.swapaxes(scale, -1, -2)
    lead = codes.shape[:-2]
    return np.concatenate([_pack(codes).reshape(*lead, -1), np.ascontiguousarray(scale).reshape(*lead, -1)], -1)


def mx4_unblocks(x, d, values):
    lead, n = x.shape[:-1], BLOCK * d // 2
    codes, scale = _unpack(x[..., :n].reshape(*lead, -1)), x[..., n:]
    if values:
        return (np.swapaxes(codes.reshape(*lead, d, BLOCK), -1, -2).copy(),
                np.swapaxes(scale.reshape(*lead, d // GROUP, BLOCK), -1, -2).copy())
    return codes.reshape(*lead, BLOCK, d).copy(), scale.reshape(*lead, BLOCK, d // GROUP).copy()


def cache_values(kind, cache, scale, d, values):
    """float64 [n][hkv][16][d] values of whole blocks in storage form (bf16: uint16 bits)."""
    if kind == "mx4":
        codes, s = mx4_unblocks(cache, d, values)
        table = np.array([e2m1_value(c) for c in range(16)])
        with np.errstate(invalid="ignore"):
            return table[codes] * np.repeat(e8m0_value(s), GROUP, -1)
    if kind == "fp8":
        with np.errstate(invalid="ignore"):
            v = e4m3_table()[cache].astype(np.float64) * scale.astype(np.float64)[:, None, None, None]
    elif kind == "bf16":
        v = (cache.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    else:
        v = cache.astype(np.float64)
    return np.swapaxes(v, -1, -2) if values else v


def rope(x, cos, sin, interleaved, exact=False):
    """x [..., d] rotated by cos, sin [..., rot / 2] (broadcast against x's leading dims)."""
    t = np.float64 if exact else np.float32
    y = np.array(x, t)
    rot = 2 * cos.shape[-1]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    u, v, c, s = np.array(x[..., a], t), np.array(x[..., b], t), np.asarray(cos, t), np.asarray(sin, t)
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., a] = u * c - v * s
        y[..., b] = v * c + u * s
    return y


def append_chunk(kind, cache, scale, table, length, rows, values, num_blocks=None, stored=None):
    """In place: rows float32 [n][hkv][d] (rotated) as the last n of `length` tokens. stored[i]: whether token i is
    stored. Blocks whose index or id is out of range store nothing."""
    nb = cache.shape[0] if num_blocks is None else num_blocks
    n, hkv, d = rows.shape
    start = length - n
    for lb in range(start // BLOCK, -(-length // BLOCK)):
        if lb >= len(table) or not 0 <= int(table[lb]) < nb:
            continue
        p = int(table[lb])
        t0, t1 = max(start, lb * BLOCK), min(length, (lb + 1) * BLOCK)
        toks = [t for t in range(t0, t1) if stored is None or stored[t - start]]
        if not toks:
            continue
        x = rows[[t - start for t in toks]]
        slots = [t % BLOCK for t in toks]
        if kind == "mx4":
            codes, s = mx4_unblocks(cache[p], d, values)
            c, e = mx4_quantise(x)
            codes[:, slots], s[:, slots] = np.swapaxes(c, 0, 1), np.swapaxes(e, 0, 1)
            cache[p] = mx4_blocks(codes, s, values)
            continue
        if kind == "fp8":
            f448, old = np.float32(448.0), np.float32(scale[p])
            top = np.float32(np.max(np.abs(x)))
            now = old
            if t0 % BLOCK == 0:
                now = np.float32(top / f448) if top > 0 else np.float32(1.0)
            elif top > np.float32(f448 * old):
                now = np.float32(top / f448)
                early = np.s_[p, :, :, :t0 % BLOCK] if values else np.s_[p, :, :t0 % BLOCK]
                dec = e4m3_table()[cache[early]].astype(np.float32)
                cache[early] = e4m3_encode(dec * old / now)
            scale[p] = now
            x = e4m3_encode(x / now)
        elif kind == "bf16":
            u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
            x = ((u + 0x7FFF + (u >> 16 & 1)) >> 16).astype(np.uint16)  # nearest, ties to even (no NaN in the tests)
        for i, slot in enumerate(slots):
            if values:
                cache[p, :, :, slot] = x[i]
            else:
                cache[p, :, slot] = x[i]


def chunk_attention(q, k, v, n, scale):
    """q [n][hq][d], k and v [hkv][length][d], all float64: (out [n][hq][d], sum of p |v|, sum of p max |v|
    [n][hq][1]) of the last n tokens, causal."""
    hkv, length, d = k.shape
    g = q.shape[1] // hkv
    out, bound, most = np.zeros(q.shape), np.zeros(q.shape), np.zeros((*q.shape[:2], 1))
    for i in range(n):
        seen = length - n + i + 1
        for h in range(q.shape[1]):
            s = k[h // g, :seen] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ v[h // g, :seen]
            bound[i, h] = p @ np.abs(v[h // g, :seen])
            most[i, h] = p @ np.abs(v[h // g, :seen]).max(1)
    return out, bound, most
