"""What the binding refuses of the tensors that a layer's products, norm and appends are given (CPU: nothing is launched)."""

import pytest
import torch

from paper_2509_00195_amd import tts as T

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture
def launched(monkeypatch):
    """The entry points' arguments, in the place of their calls."""
    calls = []
    lib = T.load()

    class Spy:
        def __getattr__(self, name):
            if name == "tts_last_error":
                return getattr(lib, name)
            return lambda *a: calls.append((name, a)) or 0

    spy = Spy()
    monkeypatch.setattr(T, "load", lambda: spy)
    return calls


def _linear(t=BF16, to=BF16, kind="bf16", out_kind="bf16", **kw):
    m, k, n = 4, 64, 32
    args = dict(x=torch.zeros((m, k), dtype=t), w=torch.zeros((n, k), dtype=t), out=torch.zeros((m, n), dtype=to),
                bias=torch.zeros(n, dtype=t), residual=torch.zeros((m, n), dtype=to))
    args.update(kw)
    T.tts_linear(T.make_linear(k, n, kind, out_kind), m, **args)


def _gated(t=BF16, **kw):
    m, k, n = 4, 64, 32
    args = dict(x=torch.zeros((m, k), dtype=t), w_gate=torch.zeros((n, k), dtype=t), w_up=torch.zeros((n, k), dtype=t),
                out=torch.zeros((m, n), dtype=t), bias_gate=torch.zeros(n, dtype=t), bias_up=torch.zeros(n, dtype=t))
    args.update(kw)
    T.tts_gated_linear(T.make_linear(k, n), m, **args)


def _rms(t=BF16, kind="bf16", **kw):
    args = dict(x=torch.zeros((4, 64), dtype=t), weight=torch.zeros(64, dtype=t), out=torch.zeros((4, 64), dtype=t))
    args.update(kw)
    T.tts_rms_norm(T.make_norm(64, 1e-6, kind, kind), 4, **args)


def test_tensors_of_the_calls_types_pass(launched):
    _linear()
    _linear(F32, BF16, "f32", "bf16")
    _linear(BF16, F32, "bf16", "f32")
    _gated()
    _rms()
    _rms(F32, "f32")
    # (Elements as bits, longer vectors, none.)
    _linear(torch.int16, torch.int16)
    _linear(bias=torch.zeros(40, dtype=BF16))
    _rms(weight=None)
    assert len(launched) == 9


@pytest.mark.parametrize("t", [F32, torch.float64, F16])
def test_vectors_of_another_type(launched, t):
    """A weight in 32 bits beside rows of bf16 holds bytes enough, but is not what the call reads."""
    with pytest.raises(ValueError, match="bias"):
        _linear(bias=torch.zeros(32, dtype=t))
    for name in ("bias_gate", "bias_up"):
        with pytest.raises(ValueError, match=name):
            _gated(**{name: torch.zeros(32, dtype=t)})
    with pytest.raises(ValueError, match="weight"):
        _rms(weight=torch.zeros(64, dtype=t))
    assert not launched


def test_vectors_of_32_bits_are_refused_others(launched):
    with pytest.raises(ValueError, match="bias"):
        _linear(F32, F32, "f32", "f32", bias=torch.zeros(64, dtype=BF16))
    with pytest.raises(ValueError, match="weight"):
        _rms(F32, "f32", weight=torch.zeros(128, dtype=BF16))
    assert not launched


def test_half_precision_is_not_bf16(launched):
    for name, shape in (("x", (4, 64)), ("w", (32, 64)), ("out", (4, 32)), ("residual", (4, 32))):
        with pytest.raises(ValueError, match=name):
            _linear(**{name: torch.zeros(shape, dtype=F16)})
    for name in ("w_gate", "w_up"):
        with pytest.raises(ValueError, match=name):
            _gated(**{name: torch.zeros((32, 64), dtype=F16)})
    for name in ("x", "out"):
        with pytest.raises(ValueError, match=name):
            _rms(**{name: torch.zeros((4, 64), dtype=F16)})
    assert not launched


def _append(norm, d=64, t=BF16, kind="bf16"):
    hq, hkv, n = 4, 2, 3
    x = torch.zeros((n, hq + 2 * hkv, d), dtype=t)
    a = 1 << 20
    T.tts_norm_rope_append_kv(T.make_desc(hq, hkv, d, q_dtype=kind, kv_dtype=kind), norm, n, n, x[:, hq:hq + hkv],
                              x[:, hq + hkv:], a, 4, a, 8, a, a, q=x[:, :hq], q_out=torch.zeros((n, hq, d), dtype=t))


@pytest.mark.parametrize("which", ["q_weight", "k_weight"])
def test_head_norm_weights_of_another_size_or_type(launched, which):
    """A weight of too few elements would be read past its end."""
    for w in (torch.zeros(63, dtype=BF16), torch.zeros(64, dtype=F32), torch.zeros(64, dtype=F16)):
        with pytest.raises(ValueError, match=which):
            _append(T.make_head_norm(**{which: w}))
    with pytest.raises(ValueError, match=which):
        _append(T.make_head_norm(**{which: torch.zeros(64, dtype=BF16)}), d=128)
    for w in (torch.zeros(64, dtype=BF16), torch.zeros(128, dtype=BF16)):
        with pytest.raises(ValueError, match=which):
            _append(T.make_head_norm(**{which: w}), t=F32, kind="f32")
    assert not launched


def test_head_norm_weights_that_fit(launched):
    _append(T.make_head_norm(torch.zeros(64, dtype=BF16), torch.zeros(72, dtype=BF16)))
    _append(T.make_head_norm(torch.zeros(64), None), t=F32, kind="f32")
    _append(T.make_head_norm())
    _append(T.make_head_norm(1 << 20, 1 << 20))  # (addresses are the caller's)
    _append(T.tts_head_norm_desc(1e-6, None, None))
    assert len(launched) == 5


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("which", ["q", "k_new", "v_new", "q_out"])
def test_appended_rows_of_another_type(launched, norm, which):
    """fp16 rows are as wide as bf16 ones, and are not what either append reads; nor do queries go into another float."""
    hq, hkv, d, n, a = 4, 2, 64, 3, 1 << 20
    args = dict(q=torch.zeros((n, hq, d), dtype=BF16), k_new=torch.zeros((n, hkv, d), dtype=BF16),
                v_new=torch.zeros((n, hkv, d), dtype=BF16), q_out=torch.zeros((n, hq, d), dtype=BF16))
    desc = T.make_desc(hq, hkv, d)

    def call(x):
        rest = dict(k_new=x["k_new"], v_new=x["v_new"], block_tables=a, max_blocks_per_seq=4, seq_lens=a, num_blocks=8,
                    k_cache=a, v_cache=a, q=x["q"], q_out=x["q_out"], rope=T.tts_rope_desc(64, 0, 16, a, a))
        if norm:
            T.tts_norm_rope_append_kv(desc, T.make_head_norm(), n, n, **rest)
        else:
            T.tts_rope_append_kv(desc, n, n, **rest)

    call(args)
    call({k: x.view(torch.int16) for k, x in args.items()})
    assert len(launched) == 2
    with pytest.raises(ValueError):
        call({**args, which: args[which].half()})
    if which == "q_out":
        with pytest.raises(ValueError):
            call({**args, which: args[which].float()})
    assert len(launched) == 2


def test_more_rows_than_an_int32_holds(launched):
    """2^32 + 1 rows would be passed on as one."""
    n = (1 << 32) + 1
    x = torch.empty((n, 1), dtype=BF16, device="meta")
    w = torch.zeros((1, 1), dtype=BF16)
    for call in (lambda: T.tts_linear(T.make_linear(1, 1), n, x, w, x), lambda: T.tts_rms_norm(T.make_norm(1), n, x, None, x),
                 lambda: T.tts_gated_linear(T.make_linear(1, 1), n, x, w, w, x)):
        with pytest.raises(ValueError, match="rows"):
            call()
    assert not launched
    T.tts_rms_norm(T.make_norm(1), (1 << 31) - 1, x, None, x)
    assert launched[0][1][1] == (1 << 31) - 1
