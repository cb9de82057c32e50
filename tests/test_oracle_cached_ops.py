"""Pins of the oracle of the operators around cached attention (CPU)."""

import numpy as np
import torch

from oracle.cached_ops import (E2M1, cache_values, chunk_attention, e2m1_value, e8m0_value, mx4_blocks, mx4_quantise,
                               mx4_unblocks, rope)


def test_e2m1_table_and_e8m0():
    assert [e2m1_value(c) for c in range(8)] == E2M1.tolist()
    assert [e2m1_value(c) for c in range(9, 16)] == (-E2M1[1:]).tolist()
    assert e8m0_value(127) == 1 and e8m0_value(0) == 2.0 ** -127 and e8m0_value(254) == 2.0 ** 127
    assert np.isnan(e8m0_value(255))


def test_quantise_hand_examples():
    x = np.zeros((1, 64), np.float32)
    # largest 7: scale 1; ties 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5 go to the even code, 7 saturates at 6
    x[0, :10] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.26, 5.01]
    codes, byte = mx4_quantise(x)
    assert byte[0, 0] == 127 and byte[0, 1] == 1
    assert codes[0, :10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9, 7]
    codes, byte = mx4_quantise(2.0 ** -9 * x)
    assert byte[0, 0] == 118 and codes[0, :10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9, 7]
    x[0, 40] = np.inf
    codes, byte = mx4_quantise(x)
    assert byte[0].tolist() == [127, 255] and (codes[0, 32:] == 0).all()
    # every E2M1 value times a power of two comes back as it is
    y = np.array([e2m1_value(c) for c in range(16)] * 2, np.float32) * np.float32(2.0 ** 5)
    codes, byte = mx4_quantise(y)
    table = np.array([e2m1_value(c) for c in range(16)])
    assert np.array_equal(table[codes] * e8m0_value(byte)[0], y)


def test_storage_round_trip_and_bytes():
    rng = np.random.default_rng(0)
    codes = rng.integers(0, 16, (3, 2, 16, 64), dtype=np.uint8)
    scale = rng.integers(100, 140, (3, 2, 16, 2), dtype=np.uint8)
    for values in (False, True):
        b = mx4_blocks(codes, scale, values)
        assert b.shape == (3, 2, 17 * 64 // 2)
        c, s = mx4_unblocks(b, 64, values)
        assert np.array_equal(c, codes) and np.array_equal(s, scale)
        # token 5, dim 42: keys token-major, values dim-major, the lower half first
        at = 5 * 64 + 42 if not values else 42 * 16 + 5
        assert (b[1, 1, at // 2] >> 4 * (at % 2)) & 15 == codes[1, 1, 5, 42]
        at = 16 * 32 + (5 * 2 + 1 if not values else 16 + 5)
        assert b[1, 1, at] == scale[1, 1, 5, 1]
        assert cache_values("mx4", b, None, 64, values)[1, 1, 5, 42] == (
            e2m1_value(int(codes[1, 1, 5, 42])) * 2.0 ** (int(scale[1, 1, 5, 1]) - 127))


def test_rope_is_a_complex_product():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 3, 64))
    angle = rng.uniform(0, 6, (4, 1, 12))
    turn = np.exp(1j * angle)
    for inter in (False, True):
        y = rope(x, np.cos(angle), np.sin(angle), inter, exact=True)
        z = (x[..., 0:24:2] + 1j * x[..., 1:24:2] if inter else x[..., :12] + 1j * x[..., 12:24]) * turn
        got = y[..., 0:24:2] + 1j * y[..., 1:24:2] if inter else y[..., :12] + 1j * y[..., 12:24]
        assert np.allclose(got, z, rtol=0, atol=1e-14) and np.array_equal(y[..., 24:], x[..., 24:])


def test_chunk_attention_against_torch():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 6, 64)), rng.standard_normal((2, 19, 64)), rng.standard_normal((2, 19, 64))
    out, bound, most = chunk_attention(q, k, v, 5, 0.125)
    t = lambda x: torch.from_numpy(x)  # noqa: E731
    mask = torch.arange(19)[None] <= torch.arange(14, 19)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(
        t(q).transpose(0, 1)[None], t(k).repeat_interleave(3, 0)[None], t(v).repeat_interleave(3, 0)[None],
        attn_mask=mask, scale=0.125)[0].transpose(0, 1).numpy()
    assert np.allclose(out, want, rtol=0, atol=1e-13) and (bound >= np.abs(out)).all() and (most >= bound).all()
