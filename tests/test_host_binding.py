"""Checks of the binding on tensors (CPU: nothing is launched)."""

import pytest
import torch

from paper_2509_00195_amd import tts as T

A = 1 << 20  # an address that no refused call reads


def _append(n=4, q=None, k=None, v=None, q_out=None, kind="bf16"):
    """A call that the library itself refuses (no tables), unless the binding does so first."""
    wide = torch.float32 if kind == "f32" else torch.bfloat16
    rows = lambda heads, m=n: torch.zeros((m, heads, 64), dtype=wide)  # noqa: E731
    desc = T.make_desc(8, 2, 64, 16, "f32" if kind == "f32" else "bf16", kind)
    T.tts_rope_append_kv(desc, 4, n, rows(2) if k is None else k, rows(2) if v is None else v, None, 4, A, 8, A, A,
                         rope=T.tts_rope_desc(64, 0, 16, A, A), q=rows(8) if q is None else q,
                         q_out=rows(8) if q_out is None else q_out)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx4"])
def test_append_refuses_tensors_of_fewer_tokens(kind):
    wide, other = (torch.float32, torch.bfloat16) if kind == "f32" else (torch.bfloat16, torch.float32)
    with pytest.raises(T.TTSError):
        _append(kind=kind)
    with pytest.raises(T.TTSError):  # more than num_tokens: padded rows
        _append(k=torch.zeros((9, 2, 64), dtype=wide), kind=kind)
    for name, heads in (("q", 8), ("k", 2), ("v", 2), ("q_out", 8)):
        with pytest.raises(ValueError):
            _append(**{name: torch.zeros((3, heads, 64), dtype=wide)}, kind=kind)
    for name, heads in (("q", 8), ("k", 2), ("v", 2)):
        with pytest.raises(ValueError):
            _append(**{name: torch.zeros((4, heads, 64), dtype=other)}, kind=kind)


def test_rows_of_one_head():
    """The stride of a dimension of size 1 says nothing: a [1][tokens][64] projection, transposed."""
    x = torch.zeros((1, 5, 64), dtype=torch.bfloat16).transpose(0, 1)
    assert x.stride(1) != 64
    assert T._rows(x, 1, 64) == (x.data_ptr(), 64)
    y = torch.zeros((2, 5, 64), dtype=torch.bfloat16).transpose(0, 1)
    with pytest.raises(ValueError):
        T._rows(y, 2, 64)


def test_an_empty_append_takes_null():
    """As the other calls do."""
    desc = T.make_desc(8, 2, 64)
    T.tts_append_kv(desc, 0, None, None, None, 0, None, 0, None, None)
    T.tts_rope_append_kv(desc, 0, 0, None, None, None, 0, None, 0, None, None)
    T.tts_rope_append_kv(desc, 3, 0, None, None, A, 4, A, 8, A, A, tok_offsets=A)


@pytest.mark.parametrize("kind,out_t", [("f32", "f32"), ("bf16", "f32"), ("fp8", "bf16")])
def test_prefill_refuses_tensors_of_fewer_tokens(kind, out_t):
    desc = T.make_desc(8, 2, 64, 16, "f32" if kind == "f32" else "bf16", kind, out_t)
    wide = torch.float32 if kind == "f32" else torch.bfloat16
    out = torch.float32 if out_t == "f32" else torch.bfloat16
    scale = A if kind == "fp8" else None

    def call(nq, no):
        """The library itself refuses the call (no tables)."""
        T.tts_paged_prefill_attn(desc, 2, 40, A, torch.zeros((nq, 8, 64), dtype=wide), A, A, scale, scale, None, 64, A, 1000, 200,
                                 torch.zeros((no, 8, 64), dtype=out), A, 1 << 40)

    for nq, no in ((40, 40), (45, 41)):
        with pytest.raises(T.TTSError):
            call(nq, no)
    for nq, no in ((39, 40), (40, 39)):
        with pytest.raises(ValueError):
            call(nq, no)
