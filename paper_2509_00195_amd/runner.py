"""Convenience callers of the C ABI for device-resident inputs.

They allocate the output and the workspace once (PyTorch allocations) and
forward every call to libtts; no arithmetic happens here. Inputs are any
object with the fields ``q, k_cache, v_cache, k_scale, v_scale,
block_tables, seq_lens`` (device tensors) plus a ``shape`` carrying
``num_q_heads, num_kv_heads, head_dim, block_size, q_dtype, kv_dtype``.
"""

from __future__ import annotations

from contextlib import nullcontext
from typing import Optional

import numpy as np
import torch

from . import tts as _t


def desc_for(shape, scale: float = 0.0) -> _t.tts_attn_desc:
    return _t.make_desc(shape.num_q_heads, shape.num_kv_heads, shape.head_dim, shape.block_size, shape.q_dtype,
                        shape.kv_dtype, "f32", scale)


class PagedAttention:
    """``tts_paged_decode_attn`` on fixed device inputs."""

    def __init__(self, inputs, max_seq_len: int, num_blocks: int, scale: float = 0.0):
        self.x = inputs
        self.desc = desc_for(inputs.shape, scale)
        self.max_seq_len = int(max_seq_len)
        self.num_blocks = int(num_blocks)
        s = int(inputs.seq_lens.shape[0])
        dev = inputs.q.device
        self.out = torch.empty((s, inputs.shape.num_q_heads, inputs.shape.head_dim), dtype=torch.float32, device=dev)
        self.ws_bytes = _t.tts_paged_decode_workspace_size(self.desc, s, self.max_seq_len)
        self.ws = torch.zeros(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)  # partial softmax states

    def __call__(self, k_cache=None, v_cache=None, k_scale=None, v_scale=None, out=None, stream=None):
        x = self.x
        o = self.out if out is None else out
        _t.tts_paged_decode_attn(
            self.desc, int(x.seq_lens.shape[0]), x.q, x.k_cache if k_cache is None else k_cache,
            x.v_cache if v_cache is None else v_cache, x.k_scale if k_scale is None else k_scale,
            x.v_scale if v_scale is None else v_scale, x.block_tables, int(x.block_tables.shape[1]), x.seq_lens,
            self.max_seq_len, self.num_blocks, o, self.ws, self.ws_bytes, stream)
        return o


class PrefixAttention:
    """``tts_build_prefix_meta`` once, then ``tts_prefix_decode_attn`` per call."""

    def __init__(self, inputs, req_seq_offsets, block_tables_host, seq_lens_host, num_blocks: int,
                 scale: float = 0.0, stream=None):
        self.x = inputs
        self.desc = desc_for(inputs.shape, scale)
        self.num_blocks = int(num_blocks)
        self.meta = _t.tts_build_prefix_meta(np.asarray(req_seq_offsets), np.asarray(block_tables_host),
                                             np.asarray(seq_lens_host), inputs.shape.block_size, self.num_blocks,
                                             desc=self.desc, stream=stream)
        s = int(inputs.seq_lens.shape[0])
        dev = inputs.q.device
        self.out = torch.empty((s, inputs.shape.num_q_heads, inputs.shape.head_dim), dtype=torch.float32, device=dev)
        self.ws_bytes = _t.tts_prefix_decode_workspace_size(self.desc, self.meta)
        self.ws = torch.zeros(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)  # partial softmax states

    def __call__(self, k_cache=None, v_cache=None, k_scale=None, v_scale=None, out=None,
                 seq_lens: Optional[torch.Tensor] = None, stream=None):
        x = self.x
        o = self.out if out is None else out
        _t.tts_prefix_decode_attn(
            self.desc, self.meta, x.q, x.k_cache if k_cache is None else k_cache,
            x.v_cache if v_cache is None else v_cache, x.k_scale if k_scale is None else k_scale,
            x.v_scale if v_scale is None else v_scale, x.block_tables, int(x.block_tables.shape[1]),
            x.seq_lens if seq_lens is None else seq_lens, self.num_blocks, o, self.ws, self.ws_bytes, stream)
        return o


def _on(stream, device):
    """The context that makes a call's stream (a handle, what has one as the calls take it, or None) the current one."""
    if stream is None:
        return nullcontext()
    handle = stream if isinstance(stream, int) else stream.cuda_stream
    return torch.cuda.stream(torch.cuda.ExternalStream(handle, device=device))


def _capturing() -> bool:
    return torch.cuda.is_available() and torch.cuda.is_current_stream_capturing()


class DecoderLayer:
    """One decoder layer over a paged cache: norm, projections, head norms with rotation and append, attention, output
    projection with its residual, norm, gated product, last projection with its residual. Every step is one call of
    libtts on buffers that are allocated once.

    ``weights``: a mapping of device tensors in the queries' type: ``attn_norm`` [hidden], ``qkv`` [(Hq + 2 Hkv) D][hidden],
    ``out`` [hidden][Hq D], ``ffn_norm`` [hidden], ``gate`` and ``up`` [ffn][hidden], ``down`` [hidden][ffn], and if
    wanted ``qkv_bias``, ``q_norm`` and ``k_norm`` [D] (without both, heads are not normalised). ``desc``: its output is of
    the queries' type."""

    def __init__(self, desc: _t.tts_attn_desc, weights, rope: _t.tts_rope_desc, max_tokens: int, max_seqs: int,
                 max_seq_len: int, num_blocks: int, eps: float = 1e-6, act: str = "silu"):
        if desc.out_dtype != desc.q_dtype:
            raise ValueError("the attention's output must be of the queries' type")
        w = self.w = dict(weights)
        self.desc, self.rope, self.max_seq_len, self.num_blocks = desc, rope, int(max_seq_len), int(num_blocks)
        self.max_seqs = int(max_seqs)
        hq, hkv, d, t = desc.num_q_heads, desc.num_kv_heads, desc.head_dim, desc.q_dtype
        for name in ("qkv", "gate"):
            if w[name].dim() != 2:
                raise ValueError(f"{name}: expected a matrix, got {tuple(w[name].shape)}")
        hidden, ffn = int(w["qkv"].shape[1]), int(w["gate"].shape[0])
        for name, rows, cols in (("qkv", (hq + 2 * hkv) * d, hidden), ("out", hidden, hq * d), ("gate", ffn, hidden),
                                 ("up", ffn, hidden), ("down", hidden, ffn)):
            _t._matrix(w[name], rows, cols, t, name)
        if _t._matrix(w["gate"], ffn, hidden, t, "gate")[1] != _t._matrix(w["up"], ffn, hidden, t, "up")[1]:
            raise ValueError("gate and up must have one row stride")
        for name in ("attn_norm", "ffn_norm"):
            _t._vector(w[name], hidden, t, name)
        for name, size in (("qkv_bias", (hq + 2 * hkv) * d), ("q_norm", d), ("k_norm", d)):
            _t._vector(w.get(name), size, t, name)
        dev, torch_t = w["qkv"].device, torch.float32 if t == _t.TTS_F32 else torch.bfloat16
        empty = lambda *shape: torch.empty(shape, dtype=torch_t, device=dev)  # noqa: E731
        self.normed, self.qkv = empty(max_tokens, hidden), empty(max_tokens, hq + 2 * hkv, d)
        self.q, self.o, self.ffn = empty(max_tokens, hq, d), empty(max_tokens, hq, d), empty(max_tokens, ffn)
        self.norm = _t.make_norm(hidden, eps, t, t)
        self.heads = None
        if w.get("q_norm") is not None or w.get("k_norm") is not None:
            self.heads = _t.make_head_norm(w.get("q_norm"), w.get("k_norm"), eps)
        self.lin_qkv = _t.make_linear(hidden, (hq + 2 * hkv) * d, t, t)
        self.lin_out = _t.make_linear(hq * d, hidden, t, t)
        self.lin_ffn = _t.make_linear(hidden, ffn, t, t, act)
        self.lin_down = _t.make_linear(ffn, hidden, t, t)
        size = max(_t.tts_linear_workspace_size(x, max_tokens) for x in (self.lin_qkv, self.lin_out, self.lin_down))
        size = max(size, _t.tts_gated_linear_workspace_size(self.lin_ffn, max_tokens),
                   _t.tts_paged_decode_workspace_size(desc, max_seqs, self.max_seq_len),
                   _t.tts_paged_prefill_workspace_size(desc, max_seqs, max_tokens, self.max_seq_len))
        self.ws = torch.empty(max(size, 1), dtype=torch.uint8, device=dev)
        self.outgrown = []  # (graphs that were captured with them, and calls under way, still write to them)
        if dev.type == "cuda" and not _capturing():
            # The buffers are the current stream's memory, where what had it before may be under way; a call may be on
            # another stream.
            torch.cuda.current_stream(dev).synchronize()

    def __call__(self, x, k_cache, v_cache, block_tables, seq_lens, k_scale=None, v_scale=None, tok_offsets=None,
                 meta: Optional[_t.PrefixMeta] = None, stream=None):
        """x [tokens][hidden], replaced by the layer's output. Without ``tok_offsets`` every sequence has one new token,
        and the attention is the paged call, or with ``meta`` the prefix-shared one; else it is the prefill, which takes no
        ``meta`` (one that is given is not used). Sizes that do not fit together are refused before anything is launched:
        a call that has appended is not to be repeated. Tokens behind the last offset (padded batches) reach no other row
        and no cache; their own rows of x hold no result. A call that needs a larger workspace than the calls before it
        allocates one: make it once before capturing it (a captured one raises). Calls of one layer, replayed ones too,
        must not overlap in time, since they share its buffers; the layer outlives them."""
        w, ws, n, s = self.w, self.ws, int(x.shape[0]), int(seq_lens.shape[0])
        hq, hkv, d = self.desc.num_q_heads, self.desc.num_kv_heads, self.desc.head_dim
        cols, cache, scales = int(block_tables.shape[1]), (k_cache, v_cache), (k_scale, v_scale)
        need = 0
        if n > self.normed.shape[0]:
            raise ValueError(f"{n} tokens in a layer made for {self.normed.shape[0]}")
        if int(block_tables.shape[0]) < s:
            raise ValueError(f"block_tables of {int(block_tables.shape[0])} sequences for {s}")
        if tok_offsets is not None:
            if not isinstance(tok_offsets, int) and int(tok_offsets.shape[0]) <= s:
                raise ValueError(f"tok_offsets has {int(tok_offsets.shape[0])} elements, {s} sequences need {s + 1}")
            need = _t.tts_paged_prefill_workspace_size(self.desc, s, n, self.max_seq_len)
        elif n != s:
            raise ValueError(f"{n} tokens for {s} sequences without tok_offsets")
        elif meta is not None:
            self._check_meta(meta, s, cols)
            need = _t.tts_prefix_decode_workspace_size(self.desc, meta)
        elif s > self.max_seqs:
            need = _t.tts_paged_decode_workspace_size(self.desc, s, self.max_seq_len)
        if self.max_seq_len > 16 * cols and (tok_offsets is not None or meta is None):
            raise ValueError(f"block_tables of {cols} columns for sequences of up to {self.max_seq_len} tokens")
        if need > ws.numel():
            ws = self._grow(need, stream)
        size, qkv, q, o, f = ws.numel(), self.qkv[:n], self.q[:n], self.o[:n], self.ffn[:n]
        _t.tts_rms_norm(self.norm, n, x, w["attn_norm"], self.normed, stream)
        _t.tts_linear(self.lin_qkv, n, self.normed, w["qkv"], qkv.flatten(1), w.get("qkv_bias"), None, ws, size, stream)
        args = (s, n, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], block_tables, cols, seq_lens, self.num_blocks, *cache, *scales)
        kw = dict(rope=self.rope, q=qkv[:, :hq], q_out=q, tok_offsets=tok_offsets, stream=stream)
        if self.heads is not None:
            _t.tts_norm_rope_append_kv(self.desc, self.heads, *args, **kw)
        else:
            _t.tts_rope_append_kv(self.desc, *args, **kw)
        if tok_offsets is not None:
            _t.tts_paged_prefill_attn(self.desc, s, n, tok_offsets, q, *cache, *scales, block_tables, cols, seq_lens,
                                      self.max_seq_len, self.num_blocks, o, ws, size, stream)
        elif meta is not None:
            _t.tts_prefix_decode_attn(self.desc, meta, q, *cache, *scales, block_tables, cols, seq_lens, self.num_blocks, o,
                                      ws, size, stream)
        else:
            _t.tts_paged_decode_attn(self.desc, s, q, *cache, *scales, block_tables, cols, seq_lens, self.max_seq_len,
                                     self.num_blocks, o, ws, size, stream)
        _t.tts_linear(self.lin_out, n, o.flatten(1), w["out"], x, None, x, ws, size, stream)
        _t.tts_rms_norm(self.norm, n, x, w["ffn_norm"], self.normed, stream)
        _t.tts_gated_linear(self.lin_ffn, n, self.normed, w["gate"], w["up"], f, None, None, ws, size, stream)
        _t.tts_linear(self.lin_down, n, f, w["down"], x, None, x, ws, size, stream)
        return x

    def _check_meta(self, meta: _t.PrefixMeta, seqs: int, cols: int):
        """The prefix-shared call refuses most of these itself, but behind the append."""
        heads = lambda d: (d.num_q_heads, d.num_kv_heads, d.head_dim)  # noqa: E731
        if not meta.handle:
            raise ValueError("meta that has been destroyed")
        held = meta.export()["num_seqs"] if meta.num_seqs is None else meta.num_seqs
        if held != seqs:
            raise ValueError(f"meta of {held} sequences for {seqs}")
        if meta.q_len != 1:
            raise ValueError("meta of a verification: a layer's step has one token for each sequence")
        if meta.desc is None or heads(meta.desc) != heads(self.desc):
            raise ValueError("meta made without a desc, or for other heads than the layer's")
        if (meta.max_blocks or cols) != cols or (meta.num_blocks or 0) > self.num_blocks:
            raise ValueError("meta of other block tables, or of more blocks than the layer's cache has")

    def _grow(self, need: int, stream):
        """A larger workspace, of the memory that belongs to the call's stream: what another stream's work has left may
        still be in use there. It is twice as large at least, so that all that are kept are less than the last one."""
        ws, captured = self.ws, _capturing()
        with _on(stream, ws.device):
            if captured or _capturing():
                raise RuntimeError("the workspace grows with this call: make it once before capturing it")
            self.outgrown.append(ws)
            self.ws = torch.empty(max(need, 2 * ws.numel()), dtype=torch.uint8, device=ws.device)
        return self.ws
