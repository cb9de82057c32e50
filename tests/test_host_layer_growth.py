"""When and where a decoder layer allocates a larger workspace (CPU: the calls are replaced)."""

import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2509_00195_amd import runner
from paper_2509_00195_amd import tts as T
from tests.test_host_decoder_layer import HIDDEN, OFFS, ROOM, SEQS, TOKENS, _call, _layer, _short, made  # noqa: F401


@pytest.fixture
def streams(monkeypatch):
    """Streams that are only names: the current one, those that are capturing, and the one that each allocation is of."""
    state = {"now": "current", "capturing": set(), "of": []}

    @contextlib.contextmanager
    def on(stream):
        before, state["now"] = state["now"], stream
        try:
            yield
        finally:
            state["now"] = before

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: f"stream {handle}")
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["now"] in state["capturing"])
    monkeypatch.setattr(runner.torch, "empty", lambda *a, **kw: state["of"].append(state["now"]) or empty(*a, **kw))
    return state


SIDE = SimpleNamespace(cuda_stream=5)


@pytest.mark.parametrize("stream,of", [(None, "current"), (SIDE, "stream 5"), (77, "stream 77"), (0, "stream 0")])
def test_a_larger_workspace_is_of_the_calls_stream(made, streams, stream, of):
    """Memory that the current stream's work has just left may still be in use there: only a call on that stream may be
    given it."""
    layer = _layer()
    _short(layer)
    streams["of"].clear()
    _call(layer, TOKENS, tok_offsets=OFFS, stream=stream)
    assert streams["of"] == [of] and streams["now"] == "current"


@pytest.mark.parametrize("stream", [None, SIDE])
@pytest.mark.parametrize("which", ["current", "stream 5"])
def test_no_allocation_in_a_capture_on_either_stream(made, streams, stream, which):
    layer = _layer()
    _short(layer)
    streams["capturing"] = {which}
    streams["of"].clear()
    if stream is None and which == "stream 5":
        _call(layer, TOKENS, tok_offsets=OFFS)
        return
    with pytest.raises(RuntimeError, match="before capturing"):
        _call(layer, TOKENS, tok_offsets=OFFS, stream=stream)
    assert not made and not streams["of"] and streams["now"] == "current"


def test_kept_workspaces_are_bounded(made, monkeypatch):
    """A need that grows by a little from call to call: what is kept for earlier captures stays below what is used."""
    layer = _layer()
    _short(layer)
    for need in range(1000, 200000, 64):
        monkeypatch.setattr(runner._t, "tts_paged_prefill_workspace_size", lambda *a, _need=need: _need)
        _call(layer, TOKENS, tok_offsets=OFFS)
        assert layer.ws.numel() >= need
    assert sum(ws.numel() for ws in layer.outgrown) <= layer.ws.numel() < 2 * 200000 and len(layer.outgrown) < 20


def test_the_largest_prefill_has_room_from_the_start(made):
    layer = _layer()
    assert layer.ws.numel() >= T.tts_paged_prefill_workspace_size(layer.desc, SEQS, TOKENS, ROOM) > 0
    ws = layer.ws
    _call(layer, TOKENS, tok_offsets=OFFS)
    assert layer.ws is ws and not layer.outgrown


def test_more_sequences_than_the_layer_was_made_for(made):
    """A decode step of more sequences needs more partial states: they are allocated, not refused behind the append."""
    layer = _layer()
    n = SEQS + 4
    x, cache = torch.zeros((n, HIDDEN), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.bfloat16)
    layer(x, cache, cache, torch.zeros((n, ROOM // 16), dtype=torch.int32), torch.ones(n, dtype=torch.int32))
    assert layer.ws.numel() >= T.tts_paged_decode_workspace_size(layer.desc, n, ROOM) > 0
