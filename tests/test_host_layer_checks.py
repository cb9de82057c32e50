"""What a decoder layer refuses before it launches anything (CPU: the calls are replaced)."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import runner
from paper_2509_00195_amd import tts as T
from tests.test_host_decoder_layer import D, HIDDEN, HKV, HQ, OFFS, ROOM, SEQS, TOKENS, _layer, made  # noqa: F401

BLOCKS = 1024  # (the layer's)


def _meta(seqs=SEQS, blocks=BLOCKS, cols=ROOM // 16, desc=None, q_len=1):
    """Metadata of sequences of two blocks and a bit, without a device: its plan is not uploaded."""
    handle = T.tts_build_prefix_meta if q_len == 1 else lambda *a: T.tts_build_verify_meta(*a[:3], q_len, *a[3:])
    tables = np.arange(seqs * cols, dtype=np.int32).reshape(seqs, cols) % blocks
    meta = handle(np.array([0, seqs], np.int32), tables, np.full(seqs, 37, np.int32), 16, blocks)
    meta.desc = desc or T.make_desc(HQ, HKV, D, block_size=16, kv_dtype="bf16", out_dtype="bf16")
    return meta


@pytest.fixture
def prefix(made, monkeypatch):
    monkeypatch.setattr(runner._t, "tts_prefix_decode_attn", lambda *a, **kw: made.append("tts_prefix_decode_attn"))
    return made


def _call(layer, n=SEQS, s=SEQS, rows=None, cols=ROOM // 16, **kw):
    x, cache = torch.zeros((n, HIDDEN), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.bfloat16)
    tables = torch.zeros((s if rows is None else rows, cols), dtype=torch.int32)
    return layer(x, cache, cache, tables, torch.ones(s, dtype=torch.int32), **kw)


def test_metadata_of_this_batch(prefix):
    layer = _layer()
    _call(layer, meta=_meta())
    assert prefix[3] == "tts_prefix_decode_attn" and len(prefix) == 8
    _call(layer, meta=_meta(blocks=BLOCKS - 9))  # (a pool that has grown since)
    assert len(prefix) == 16


@pytest.mark.parametrize("kw", [dict(seqs=SEQS + 1), dict(seqs=SEQS - 1), dict(cols=ROOM // 16 + 1), dict(blocks=BLOCKS + 1),
                                dict(q_len=2), dict(desc=T.make_desc(HQ, HKV, 128)), dict(desc=T.make_desc(HQ, 1, D)),
                                dict(desc=T.make_desc(2 * HQ, HKV, D))])
def test_metadata_of_another_batch(prefix, kw):
    """More beams than the batch has would read lengths and tables behind their end, and write behind the layer's rows."""
    with pytest.raises(ValueError, match="meta"):
        _call(_layer(), meta=_meta(**kw))
    assert not prefix


@pytest.mark.parametrize("kw", [dict(n=SEQS + 1), dict(n=SEQS - 1), dict(rows=SEQS - 1), dict(n=TOKENS, tok_offsets=OFFS[:3]),
                                dict(n=TOKENS, tok_offsets=OFFS, rows=1)])
def test_batches_that_do_not_fit_together(made, kw):
    with pytest.raises(ValueError):
        _call(_layer(), **kw)
    assert not made


@pytest.mark.parametrize("kw", [dict(), dict(n=TOKENS, tok_offsets=OFFS)])
def test_tables_shorter_than_the_longest_sequence(made, kw):
    with pytest.raises(ValueError, match="columns"):
        _call(_layer(), cols=ROOM // 16 - 1, **kw)
    assert not made


def test_metadata_wrapped_by_hand(prefix):
    """A handle without the sizes of its batch: how many beams it is of is asked of it."""
    layer, meta = _layer(), _meta()
    _call(layer, meta=T.PrefixMeta(meta.handle, meta.desc))
    assert len(prefix) == 8
    more = _meta(seqs=SEQS + 1)
    for m in (meta, more):
        m.destroy = lambda: None
    with pytest.raises(ValueError, match="meta"):
        _call(layer, meta=T.PrefixMeta(more.handle, more.desc))
    assert len(prefix) == 8


def test_metadata_that_has_been_destroyed(prefix):
    meta = _meta()
    meta.destroy()
    with pytest.raises(ValueError, match="meta"):
        _call(_layer(), meta=meta)
    assert not prefix


def test_batches_that_do(made):
    layer = _layer()
    _call(layer, rows=SEQS + 2)
    _call(layer, n=TOKENS, tok_offsets=OFFS)
    _call(layer, n=TOKENS, tok_offsets=OFFS, meta=_meta(seqs=SEQS + 1))  # (the prefill takes no metadata)
    _call(layer, n=TOKENS, tok_offsets=1 << 20)  # (an address)
    assert len(made) == 32


def _weights(**kw):
    t = torch.bfloat16
    w = dict(attn_norm=torch.ones(HIDDEN, dtype=t), qkv=torch.ones(((HQ + 2 * HKV) * D, HIDDEN), dtype=t),
             out=torch.ones((HIDDEN, HQ * D), dtype=t), ffn_norm=torch.ones(HIDDEN, dtype=t),
             gate=torch.ones((256, HIDDEN), dtype=t), up=torch.ones((256, HIDDEN), dtype=t),
             down=torch.ones((HIDDEN, 256), dtype=t), qkv_bias=torch.ones((HQ + 2 * HKV) * D, dtype=t),
             q_norm=torch.ones(D, dtype=t), k_norm=torch.ones(D, dtype=t))
    w.update(kw)
    return w


def _made_of(w):
    desc = T.make_desc(HQ, HKV, D, block_size=16, kv_dtype="bf16", out_dtype="bf16")
    return runner.DecoderLayer(desc, w, None, TOKENS, SEQS, ROOM, BLOCKS)


@pytest.mark.parametrize("name", ["attn_norm", "qkv", "out", "ffn_norm", "gate", "up", "down", "qkv_bias", "q_norm", "k_norm"])
def test_weights_of_another_shape_or_type(name):
    """At the start, not when a call has half run: the last product's weight was looked at behind the append."""
    x = _weights()[name]
    short = x[:-1] if name != "gate" else x[:, :-1]  # (the gate's rows give the layer its width)
    for bad in (x.float(), x.half(), short):
        with pytest.raises(ValueError, match=name):
            _made_of(_weights(**{name: bad}))
    if x.dim() == 2:
        for bad in (x[:, :-1], x.t(), x.flatten()):
            with pytest.raises(ValueError):
                _made_of(_weights(**{name: bad}))


def test_weights_that_fit():
    _made_of(_weights())
    _made_of(_weights(qkv_bias=None, q_norm=None, k_norm=None))
    apart = torch.ones((256, HIDDEN + 8), dtype=torch.bfloat16)[:, :HIDDEN]
    _made_of(_weights(gate=apart, up=apart))
    with pytest.raises(ValueError, match="stride"):
        _made_of(_weights(gate=apart))
    for name in ("down", "ffn_norm"):
        w = _weights()
        del w[name]
        with pytest.raises(KeyError):
            _made_of(w)
