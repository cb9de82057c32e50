"""A decoder layer on another stream than the one its memory belongs to, and with heads of 128."""

import numpy as np
import pytest
import torch

from paper_2509_00195_amd import make_rope, tts_build_prefix_meta, tts_rope_tables
from paper_2509_00195_amd.runner import DecoderLayer
from tests import _layer as L
from tests._cached import BS, DEV, Cache, desc_of

pytestmark = pytest.mark.gpu
HQ, HKV, HIDDEN, FFN, ROOM = 4, 2, 512, 1024, 2048


class Run:
    def __init__(self, seqs, d, tokens, seed=3):
        g = L.generator(seed)
        mat = lambda n, k: L.rows((n, k), 0, "bf16", g, k ** -0.5)  # noqa: E731
        self.w = dict(attn_norm=mat(1, HIDDEN)[0].contiguous(), qkv=mat((HQ + 2 * HKV) * d, HIDDEN), out=mat(HIDDEN, HQ * d),
                      ffn_norm=mat(1, HIDDEN)[0].contiguous(), gate=mat(FFN, HIDDEN), up=mat(FFN, HIDDEN),
                      down=mat(HIDDEN, FFN), q_norm=mat(1, d)[0].contiguous())
        self.c = Cache("bf16", HKV, d, [ROOM] * seqs, np.random.default_rng(seed))
        self.dev = self.c.device()
        self.tables = torch.from_numpy(np.ascontiguousarray(self.c.tables)).to(DEV)
        self.lens = torch.full((seqs,), ROOM - 2, dtype=torch.int32, device=DEV)
        self.angles = tuple(torch.from_numpy(t).to(DEV) for t in tts_rope_tables(d, 1e4, ROOM))
        self.desc, self.tokens, self.seqs = desc_of("bf16", HQ, HKV, d, "bf16"), tokens, seqs
        self.x = torch.randn((tokens, HIDDEN), generator=g, device=DEV).to(torch.bfloat16)

    def layer(self):
        return DecoderLayer(self.desc, self.w, make_rope(*self.angles), self.tokens, self.seqs, ROOM, self.c.nb)

    def call(self, layer, x, **kw):
        return layer(x, *self.dev[:2], self.tables, self.lens, **kw)


@pytest.mark.parametrize("when", ["made", "grown"])
def test_memory_that_the_current_stream_has_just_left(when):
    """What had the memory before is still being written on the current stream when the layer is made, or grows."""
    r = Run(4, 64, 4)
    want = r.call(r.layer(), r.x.clone())
    layer, side, x = r.layer(), torch.cuda.Stream(), r.x.clone()
    if when == "grown":
        layer.ws = torch.empty(16, dtype=torch.uint8, device=DEV)
    meta = tts_build_prefix_meta(np.array([0, 4], np.int32), r.c.tables, np.full(4, ROOM - 2, np.int32), BS, r.c.nb, desc=r.desc)
    shared = r.call(r.layer(), r.x.clone(), meta=meta)
    torch.cuda.synchronize()
    junk = torch.empty(1 << 30, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for i in range(100):
        junk.fill_(255 - i % 2)
    del junk
    if when == "made":
        out, want = r.call(r.layer(), x, stream=side), want
    else:
        out, want = r.call(layer, x, stream=side, meta=meta), shared
        assert layer.ws.numel() > 16
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("d", [64, 128])
def test_a_stream_by_its_handle(d):
    r = Run(3, d, 3)
    layer, side, x = r.layer(), torch.cuda.Stream(), r.x.clone()
    layer.ws = torch.empty(16, dtype=torch.uint8, device=DEV)
    meta = tts_build_prefix_meta(np.array([0, 3], np.int32), r.c.tables, np.full(3, ROOM - 2, np.int32), BS, r.c.nb, desc=r.desc)
    shared = r.call(r.layer(), r.x.clone(), meta=meta)
    torch.cuda.synchronize()
    out = r.call(layer, x, stream=side.cuda_stream, meta=meta)
    torch.cuda.synchronize()
    assert torch.equal(out, shared)


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp8", "mx4"])
def test_prompts_then_decode_steps_of_heads_of_128(kind, monkeypatch):
    from tests import test_gpu_layer as M

    monkeypatch.setattr(M, "D", 128)
    M.test_prompts_then_decode_steps(kind, True)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_a_padded_batch(kind):
    """Rows behind the last offset reach nothing: neither the sequences' rows nor the caches depend on what they hold."""
    from tests.test_gpu_layer import HIDDEN as WIDTH
    from tests.test_gpu_layer import Model

    new = [5, 0, 20, 1]
    offs = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    found = []
    for fill in (0.0, float("nan"), float("inf"), 3.0):
        m = Model(kind, 4, 5)
        m.lens += torch.tensor([40, 7, 60, 33], dtype=torch.int32, device=DEV)
        x = torch.full((sum(new) + 6, WIDTH), fill, dtype=torch.bfloat16, device=DEV)
        x[:sum(new)] = m.hidden(sum(new))
        m.layer.o.fill_(fill)
        m.run(x, offs)
        torch.cuda.synchronize()
        found.append([x[:sum(new)].clone(), *(t.clone() for t in m.dev if t is not None)])
    assert bool(torch.isfinite(found[0][0]).all())
    for other in found[1:]:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(found[0], other))
