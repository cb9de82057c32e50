"""Refusals, sizes and plans of a layer's products, norm and append with head norms (CPU: nothing is launched)."""

import ctypes as C

import pytest
import torch

from paper_2509_00195_amd import tts as T

A = 1 << 20  # an aligned address that no refused call reads
INV, UNS, WSP = T.TTS_ERR_INVALID_ARG, T.TTS_ERR_UNSUPPORTED, T.TTS_ERR_WORKSPACE


def _status(call, *args, **kw):
    with pytest.raises(T.TTSError) as e:
        call(*args, **kw)
    return e.value.status


def _linear(k=64, n=32, m=4, x=A, xs=None, w=A, ws=None, bias=None, res=None, rs=None, out=A, os_=None, work=None, size=0,
            dtype="bf16", out_dtype="bf16", act="none"):
    d = T.make_linear(k, n, dtype, out_dtype, act)
    return T.load().tts_linear(C.byref(d), m, x, k if xs is None else xs, w, k if ws is None else ws, bias, res,
                               n if rs is None else rs, out, n if os_ is None else os_, work, size, None)


def _gated(k=64, n=32, m=4, x=A, xs=None, w=A, u=A, ws=None, b0=None, b1=None, out=A, os_=None, work=None, size=0,
           dtype="bf16", out_dtype="bf16", act="silu"):
    d = T.make_linear(k, n, dtype, out_dtype, act)
    return T.load().tts_gated_linear(C.byref(d), m, x, k if xs is None else xs, w, u, k if ws is None else ws, b0, b1, out,
                                     n if os_ is None else os_, work, size, None)


BOTH = [(dict(m=-1), INV), (dict(k=0), INV), (dict(n=0), INV), (dict(k=-4), INV), (dict(x=None), INV), (dict(w=None), INV),
        (dict(out=None), INV), (dict(xs=63), INV), (dict(ws=63), INV), (dict(os_=31), INV), (dict(xs=-64), INV),
        (dict(x=A + 1), INV), (dict(w=A + 1), INV), (dict(out=A + 1), INV), (dict(x=A + 2, dtype="f32"), INV),
        (dict(out=A + 2, out_dtype="f32"), INV), (dict(act=5), INV), (dict(act=-1), INV), (dict(dtype="fp8"), UNS),
        (dict(out_dtype="mx4"), UNS), (dict(k=(1 << 28) + 1), UNS), (dict(n=(1 << 26) + 1), UNS),
        (dict(xs=(1 << 31) + 1), UNS), (dict(ws=(1 << 31) + 1), UNS), (dict(os_=(1 << 31) + 1), UNS),
        (dict(m=(1 << 31) - 1, n=1 << 20), UNS)]


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(res=A, rs=31), INV), (dict(res=A, os_=40), INV), (dict(res=A + 1), INV), (dict(bias=A + 1), INV),
    (dict(res=A + 2, out_dtype="f32"), INV), (dict(res=2 * A, rs=(1 << 31) + 1), UNS)])
def test_linear_refusals(kw, status):
    assert _linear(**kw) == status


@pytest.mark.parametrize("kw,status", BOTH + [(dict(u=None), INV), (dict(u=A + 1), INV), (dict(b0=A + 1), INV),
                                              (dict(b1=A + 1), INV)])
def test_gated_refusals(kw, status):
    assert _gated(**kw) == status


def test_workspaces():
    d = T.make_linear(8192, 144)
    for need, call in ((T.tts_linear_workspace_size, _linear), (T.tts_gated_linear_workspace_size, _gated)):
        size = need(d, 16)
        assert size > 0
        assert call(k=8192, n=144, m=16, work=A, size=16 * 144 * 4) == WSP  # less than one part's sums
        assert call(k=8192, n=144, m=16, work=None, size=size) == WSP
        assert call(k=8192, n=144, m=16, work=A + 8, size=size) == INV
        assert need(d, 0) == 0 and need(d, -3) == 0
        assert need(T.make_linear(64, 144), 16) == 0  # too short to split
        sizes = [need(d, m) for m in (1, 2, 16, 17, 33, 64, 65, 128, 129, 300, 1000, 1 << 20, 1 << 30)]
        assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]  # large calls are not split
    assert T.tts_linear_workspace_size(T.make_linear(0, 144), 16) == 0


def test_a_null_desc():
    lib = T.load()
    assert lib.tts_linear(None, 1, A, 64, A, 64, None, None, 0, A, 64, None, 0, None) == INV
    assert lib.tts_gated_linear(None, 1, A, 64, A, A, 64, None, None, A, 64, None, 0, None) == INV
    assert lib.tts_rms_norm(None, 1, A, 64, None, A, 64, None) == INV
    assert lib.tts_linear_workspace_size(None, 4) == 0


def _rms(k=64, m=4, x=A, xs=None, w=None, out=2 * A, os_=None, eps=1e-6, dtype="bf16", out_dtype="bf16"):
    d = T.make_norm(k, eps, dtype, out_dtype)
    return T.load().tts_rms_norm(C.byref(d), m, x, k if xs is None else xs, w, out, k if os_ is None else os_, None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), INV), (dict(k=-1), INV), (dict(m=-1), INV), (dict(x=None), INV), (dict(out=None), INV), (dict(xs=63), INV),
    (dict(os_=63), INV), (dict(x=A + 1), INV), (dict(w=A + 1), INV), (dict(out=A + 1), INV), (dict(eps=-1e-6), INV),
    (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV), (dict(out=A, os_=72), INV),
    (dict(out=A, out_dtype="f32"), INV), (dict(dtype="fp8"), UNS), (dict(out_dtype="fp8"), UNS), (dict(xs=(1 << 31) + 1), UNS)])
def test_rms_refusals(kw, status):
    assert _rms(**kw) == status


def test_no_rows():
    assert _linear(m=0, x=None, w=None, out=None) == T.TTS_OK
    assert _gated(m=0, x=None, w=None, u=None, out=None) == T.TTS_OK
    assert _rms(m=0, x=None, out=None) == T.TTS_OK


def _append(norm=T.tts_head_norm_desc(1e-6, None, None), desc=None, rope=None, s=2, n=2, k=A, v=A, tables=A, cols=4, lens=A,
            nb=8, kc=A, vc=A, **kw):
    T.tts_norm_rope_append_kv(desc or T.make_desc(8, 2, 64), norm, s, n, k, v, tables, cols, lens, nb, kc, vc, rope=rope, **kw)


def _rope(rot=64, inter=0, most=16, cos=A, sin=A):
    return T.tts_rope_desc(rot, inter, most, cos, sin)


@pytest.mark.parametrize("kw", [
    dict(norm=None), dict(norm=T.tts_head_norm_desc(-1.0, A, A)), dict(norm=T.tts_head_norm_desc(float("nan"), A, A)),
    dict(norm=T.tts_head_norm_desc(float("inf"), A, A)), dict(s=-1), dict(n=3), dict(k=None), dict(v=None), dict(tables=None),
    dict(lens=None), dict(kc=None), dict(kc=A + 8), dict(positions=A), dict(q=A), dict(q_out=A), dict(rope=_rope(63)),
    dict(rope=_rope(), q=A), dict(rope=_rope(cos=None)), dict(k_scale=A, v_scale=A),
    dict(norm=T.tts_head_norm_desc(1e-6, A + 1, None)), dict(norm=T.tts_head_norm_desc(1e-6, None, A + 1))])
def test_append_refusals(kw):
    assert _status(_append, **kw) == INV


def test_nothing_to_append_is_accepted():
    _append(s=0, n=0)
    _append(n=0, tok_offsets=A)
    _append(n=0, tok_offsets=A, q=A, q_out=2 * A)


def test_the_binding_checks_tensors():
    d = T.make_linear(64, 32)
    x, w, o = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((32, 64), dtype=torch.bfloat16), torch.zeros(
        (4, 32), dtype=torch.bfloat16)
    bad = [dict(x=x[:3]), dict(x=x.float()), dict(x=torch.zeros((4, 65), dtype=torch.bfloat16)), dict(w=w[:31]),
           dict(w=torch.zeros((64, 32), dtype=torch.bfloat16).t()), dict(out=o[:3]), dict(out=o.float()),
           dict(bias=torch.zeros(31, dtype=torch.bfloat16)), dict(residual=o[:2]), dict(residual=o.float()), dict(x=x[0])]
    for kw in bad:
        args = {"x": x, "w": w, "out": o, **kw}
        with pytest.raises(ValueError):
            T.tts_linear(d, 4, args["x"], args["w"], args["out"], args.get("bias"), args.get("residual"))
    for kw in (dict(u=torch.zeros((32, 72), dtype=torch.bfloat16)[:, :64]), dict(u=w[:4]), dict(b=torch.zeros(3))):
        with pytest.raises(ValueError):
            T.tts_gated_linear(d, 4, x, w, kw.get("u", w), o, None, kw.get("b"))
    n = T.make_norm(64)
    for args in ((x.float(), None, x), (x, None, x[:3]), (x, torch.zeros(63, dtype=torch.bfloat16), x)):
        with pytest.raises(ValueError):
            T.tts_rms_norm(n, 4, *args)
    assert T._matrix(x[:1, :], 1, 64, T.TTS_BF16, "x")[1] == 64
    assert T._matrix(torch.zeros((4, 80), dtype=torch.bfloat16)[:, :64], 4, 64, T.TTS_BF16, "x")[1] == 80
    assert T._matrix(torch.zeros((4, 1), dtype=torch.bfloat16), 4, 1, T.TTS_BF16, "x")[1] == 1
