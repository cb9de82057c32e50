"""A decoder layer's buffers: what its calls are given, without a device."""

import weakref

import pytest
import torch

from paper_2509_00195_amd import runner
from paper_2509_00195_amd import tts as T

HQ, HKV, D, HIDDEN, FFN, SEQS, TOKENS, ROOM = 4, 2, 64, 128, 256, 3, 8, 4096
CALLS = ["tts_rms_norm", "tts_linear", "tts_gated_linear", "tts_rope_append_kv", "tts_norm_rope_append_kv",
         "tts_paged_decode_attn", "tts_paged_prefill_attn"]


@pytest.fixture
def made(monkeypatch):
    """Names of the calls that are made, which do nothing."""
    names = []
    for name in CALLS:
        monkeypatch.setattr(runner._t, name, lambda *a, _name=name, **kw: names.append(_name))
    return names


def _layer(q_norm=True):
    t = torch.bfloat16
    w = dict(attn_norm=torch.ones(HIDDEN, dtype=t), qkv=torch.ones(((HQ + 2 * HKV) * D, HIDDEN), dtype=t),
             out=torch.ones((HIDDEN, HQ * D), dtype=t), ffn_norm=torch.ones(HIDDEN, dtype=t),
             gate=torch.ones((FFN, HIDDEN), dtype=t), up=torch.ones((FFN, HIDDEN), dtype=t),
             down=torch.ones((HIDDEN, FFN), dtype=t))
    if q_norm:
        w["q_norm"] = torch.ones(D, dtype=t)
    desc = T.make_desc(HQ, HKV, D, block_size=16, kv_dtype="bf16", out_dtype="bf16")
    return runner.DecoderLayer(desc, w, None, TOKENS, SEQS, ROOM, 1024)


def _call(layer, n, **kw):
    x = torch.zeros((n, HIDDEN), dtype=torch.bfloat16)
    cache = torch.zeros(1, dtype=torch.bfloat16)
    return layer(x, cache, cache, torch.zeros((SEQS, ROOM // 16), dtype=torch.int32), torch.ones(SEQS, dtype=torch.int32), **kw)


OFFS = torch.tensor([0, 2, 4, TOKENS], dtype=torch.int32)


def _short(layer):
    """As if the calls before had needed less than the prefill does."""
    layer.ws = torch.empty(16, dtype=torch.uint8)
    return weakref.ref(layer.ws)


@pytest.mark.parametrize("q_norm", [True, False])
def test_the_calls_of_a_step(made, q_norm):
    _call(_layer(q_norm), SEQS)
    append = "tts_norm_rope_append_kv" if q_norm else "tts_rope_append_kv"
    assert made == ["tts_rms_norm", "tts_linear", append, "tts_paged_decode_attn", "tts_linear", "tts_rms_norm",
                    "tts_gated_linear", "tts_linear"]


def test_an_outgrown_workspace_lives_on(made):
    """A graph that was captured before a larger call still writes to the workspace of its own capture."""
    layer = _layer()
    old = _short(layer)
    _call(layer, TOKENS, tok_offsets=OFFS)
    need = T.tts_paged_prefill_workspace_size(layer.desc, SEQS, TOKENS, ROOM)
    assert need > 16 and layer.ws.numel() == need
    assert old() is not None


def test_a_captured_call_does_not_allocate(made, monkeypatch):
    layer = _layer()
    _short(layer)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="before capturing"):
        _call(layer, TOKENS, tok_offsets=OFFS)
    assert not made and layer.ws.numel() == 16


def test_more_tokens_than_room(made):
    with pytest.raises(ValueError, match="made for 8"):
        _call(_layer(), TOKENS + 1)
    assert not made
