"""Refusals and sizes of the operators around cached attention (CPU: nothing is launched)."""

import ctypes as C

import numpy as np
import pytest

from paper_2509_00195_amd import tts as T

A = 1 << 20  # an aligned address that no refused call reads


def _status(call, *args, **kw):
    with pytest.raises(T.TTSError) as e:
        call(*args, **kw)
    return e.value.status


def _append(desc=None, rope=None, s=2, n=2, k=A, v=A, tables=A, cols=4, lens=A, nb=8, kc=A, vc=A, **kw):
    T.tts_rope_append_kv(desc or T.make_desc(8, 2, 64), s, n, k, v, tables, cols, lens, nb, kc, vc, rope=rope, **kw)


def _rope(rot=64, inter=0, most=16, cos=A, sin=A):
    return T.tts_rope_desc(rot, inter, most, cos, sin)


@pytest.mark.parametrize("kw", [
    dict(s=-1), dict(n=-1), dict(cols=-1), dict(nb=-1), dict(n=3), dict(k=None), dict(v=None), dict(tables=None),
    dict(lens=None), dict(kc=None), dict(vc=None), dict(kc=A + 8), dict(vc=A + 4), dict(q=A, q_out=A), dict(positions=A),
    dict(rope=_rope(63)), dict(rope=_rope(66)), dict(rope=_rope(-2)), dict(rope=_rope(inter=2)), dict(rope=_rope(most=-1)),
    dict(rope=_rope(cos=None)), dict(rope=_rope(sin=None)), dict(rope=_rope(), q=A), dict(rope=_rope(), q_out=A),
    dict(k_scale=A, v_scale=A), dict(desc=T.make_desc(8, 2, 64, kv_dtype="fp8")),
    dict(desc=T.make_desc(8, 2, 64, kv_dtype="mx4"), k_scale=A, v_scale=A),
])
def test_append_refusals(kw):
    assert _status(_append, **kw) == T.TTS_ERR_INVALID_ARG


def test_append_strides_and_limits():
    lib = T.load()
    desc, rope = T.make_desc(8, 2, 64), _rope()

    def call(q, qs, ks, vs, q_out, d=desc):
        return lib.tts_rope_append_kv(C.byref(d), C.byref(rope), 2, 2, None, None, q, qs, A, ks, A, vs, A, 4, A, 8, q_out, A,
                                      A, None, None, None)

    assert call(A, 8 * 64, 127, 128, 2 * A) == T.TTS_ERR_INVALID_ARG
    assert call(A, 8 * 64, 128, 127, 2 * A) == T.TTS_ERR_INVALID_ARG
    assert call(A, 511, 128, 128, 2 * A) == T.TTS_ERR_INVALID_ARG
    assert call(A, 768, 128, 128, A) == T.TTS_ERR_INVALID_ARG  # in place with gaps
    big = T.make_desc(8256, 258, 64)
    assert lib.tts_rope_append_kv(C.byref(big), None, 2, 2, None, None, None, 0, A, 258 * 64, A, 258 * 64, A, 4, A, 8, None, A,
                                  A, None, None, None) == T.TTS_ERR_UNSUPPORTED


def test_nothing_to_do_is_accepted():
    _append(s=0, n=0)
    _append(n=0, tok_offsets=A)
    T.tts_paged_prefill_attn(T.make_desc(8, 2, 64), 0, 0, None, None, None, None, None, None, None, 0, None, 0, 0, None, None,
                             0)


def _prefill(desc=None, s=2, n=40, offs=A, q=A, k=A, v=A, ks=None, vs=None, tables=A, cols=64, lens=A, most=1000, nb=200,
             out=A, ws=A, size=1 << 40):
    T.tts_paged_prefill_attn(desc or T.make_desc(8, 2, 64), s, n, offs, q, k, v, ks, vs, tables, cols, lens, most, nb, out, ws,
                             size)


@pytest.mark.parametrize("kw", [
    dict(s=-1), dict(n=-1), dict(cols=-1), dict(most=-1), dict(nb=-1), dict(most=64 * 16 + 1), dict(offs=None), dict(q=None),
    dict(k=None), dict(v=None), dict(tables=None), dict(lens=None), dict(out=None), dict(q=A + 8), dict(k=A + 2),
    dict(v=A + 4), dict(out=A + 8), dict(ks=A, vs=A), dict(desc=T.make_desc(8, 2, 64, kv_dtype="fp8")),
    dict(desc=T.make_desc(8, 2, 64, kv_dtype="mx4"), ks=A, vs=A),
])
def test_prefill_refusals(kw):
    assert _status(_prefill, **kw) == T.TTS_ERR_INVALID_ARG


def test_prefill_workspace():
    d = T.make_desc(8, 2, 64)
    need = T.tts_paged_prefill_workspace_size(d, 2, 40, 1000)
    assert need > 0
    assert _status(_prefill, size=need - 1) == T.TTS_ERR_WORKSPACE
    assert _status(_prefill, ws=None) == T.TTS_ERR_WORKSPACE
    assert _status(_prefill, ws=A + 8) == T.TTS_ERR_INVALID_ARG  # aligned to 16 bytes
    assert T.tts_paged_prefill_workspace_size(d, 2, 40, 200) == 0  # too short to split
    assert T.tts_paged_prefill_workspace_size(d, 64, 1 << 16, 4096) == 0  # rows enough
    assert T.tts_paged_prefill_workspace_size(d, -1, 40, 1000) == 0
    assert _status(_prefill, n=(1 << 31) // 8) == T.TTS_ERR_UNSUPPORTED


def test_sequences_whose_tiles_would_pass_int32():
    most, cols = (1 << 31) - 1, 1 << 27
    assert _status(_prefill, most=most, cols=cols) == T.TTS_ERR_UNSUPPORTED
    d = T.make_desc(8, 2, 64, kv_dtype="mx4")
    assert _status(T.tts_paged_decode_attn, d, 2, A, A, A, None, None, A, cols, A, most, 8, A, A, 1 << 60) == T.TTS_ERR_UNSUPPORTED


@pytest.mark.parametrize("args", [
    dict(q_dtype="f32", kv_dtype="mx4"), dict(q_dtype="bf16", kv_dtype="f32"), dict(out_dtype=2), dict(out_dtype=3),
    dict(kv_dtype=4), dict(head_dim=96), dict(block_size=32),
])
def test_unsupported_descs(args):
    d = T.make_desc(8, 2, args.pop("head_dim", 64), args.pop("block_size", 16), **args)
    assert _status(_append, desc=d) == T.TTS_ERR_UNSUPPORTED
    assert _status(_prefill, desc=d) == T.TTS_ERR_UNSUPPORTED


def test_mx4_scales_must_be_null():
    d = T.make_desc(8, 2, 64, kv_dtype="mx4")
    assert _status(T.tts_append_kv, d, 2, A, A, A, 4, A, 8, A, A, A, A) == T.TTS_ERR_INVALID_ARG
    assert _status(T.tts_copy_blocks, d, 2, A, 8, A, A, A, A) == T.TTS_ERR_INVALID_ARG
    assert _status(T.tts_paged_decode_attn, d, 2, A, A, A, A, A, A, 4, A, 60, 8, A, A, 1 << 30) == T.TTS_ERR_INVALID_ARG


def test_rope_tables():
    cos, sin = T.tts_rope_tables(48, 1e6, 300)
    i, t = np.arange(24), np.arange(300)[:, None]
    angle = t * 1e6 ** (-i / 24.0)
    # a float of the double, whose angle (below 300) is 2^-52 of itself off: under 2^-43
    assert np.abs(cos - np.cos(angle)).max() <= 2.0 ** -25 + 2.0 ** -43
    assert np.abs(sin - np.sin(angle)).max() <= 2.0 ** -25 + 2.0 ** -43
    assert T.tts_rope_tables(0, 1e4, 5)[0].shape == (5, 0)
    for bad in ((63, 1e4, 4), (-2, 1e4, 4), (64, 0.0, 4), (64, float("nan"), 4), (64, float("inf"), 4), (64, 1e4, -1)):
        assert _status(T.tts_rope_tables, *bad) == T.TTS_ERR_INVALID_ARG


def test_binding_checks_rows_and_tables():
    import torch

    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        T._rows(x, 2, 64)
    with pytest.raises(ValueError):
        T._rows(x.transpose(0, 1), 2, 64)
    assert T._rows(x[:, 1:3], 2, 64)[1] == 4 * 64
    assert T._rows(x[:1, 1:3], 2, 64)[1] == 2 * 64
    with pytest.raises(ValueError):
        T.make_rope(torch.zeros(4, 8), torch.zeros(4, 9))
    with pytest.raises(ValueError):
        T.make_rope(torch.zeros(4, 8, dtype=torch.float64), torch.zeros(4, 8, dtype=torch.float64))
