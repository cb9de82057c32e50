"""A decoder layer's calls in a row, as a program makes them: prompts, then decode steps, eager and captured."""

import numpy as np
import pytest
import torch

from oracle.cached_ops import append_chunk, rope
from oracle.layer_ops import head_norm
from paper_2509_00195_amd import make_rope, tts_build_prefix_meta, tts_rope_tables
from paper_2509_00195_amd.runner import DecoderLayer
from tests import _layer as L
from tests._cached import BS, DEV, KINDS, Cache, close, desc_of, reference

pytestmark = pytest.mark.gpu
HQ, HKV, D, HIDDEN, FFN, ROOM, EPS = 8, 2, 64, 384, 1000, 160, 1e-6


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Model:
    def __init__(self, kind, seqs, seed, heads=True):
        self.kind, self.t = kind, "f32" if kind == "f32" else "bf16"
        self.g = L.generator(seed)
        rng = np.random.default_rng(seed)
        mat = lambda n, k: L.rows((n, k), 0, self.t, self.g, k ** -0.5)  # noqa: E731
        vec = lambda n: (1 + 0.2 * torch.randn(n, generator=self.g, device=DEV)).to(L.TYPES[self.t])  # noqa: E731
        self.w = dict(attn_norm=vec(HIDDEN), qkv=mat((HQ + 2 * HKV) * D, HIDDEN), qkv_bias=vec((HQ + 2 * HKV) * D),
                      out=mat(HIDDEN, HQ * D), ffn_norm=vec(HIDDEN), gate=mat(FFN, HIDDEN), up=mat(FFN, HIDDEN),
                      down=mat(HIDDEN, FFN))
        if heads:
            self.w.update(q_norm=vec(D), k_norm=vec(D))
        self.c = Cache(kind, HKV, D, [ROOM] * seqs, rng)
        self.c.lens = np.zeros(seqs, np.int32)
        self.dev = self.c.device()
        self.tables, self.lens = _up(self.c.tables), torch.zeros(seqs, dtype=torch.int32, device=DEV)
        self.cos, self.sin = tts_rope_tables(D, 1e4, ROOM)
        self.keep = (_up(self.cos), _up(self.sin))
        self.desc = desc_of(kind, HQ, HKV, D, self.t)
        self.layer = DecoderLayer(self.desc, self.w, make_rope(*self.keep), 300, seqs, ROOM, self.c.nb, EPS)

    def hidden(self, n):
        return torch.randn((n, HIDDEN), generator=self.g, device=DEV).to(L.TYPES[self.t])

    def run(self, x, offs=None, meta=None, stream=None):
        return self.layer(x, *self.dev[:2], self.tables, self.lens, *self.dev[2:], tok_offsets=offs, meta=meta, stream=stream)

    def check(self, x, out, new):
        """Each step against its definition, on what the step before it left."""
        w, y, n = self.w, self.layer, len(x)
        torch.cuda.synchronize()
        qkv = y.qkv[:n]
        # The norm before the projection is overwritten by the second one; it is made again, as the call makes it.
        from paper_2509_00195_amd import tts_rms_norm

        first = torch.empty_like(y.normed)
        tts_rms_norm(y.norm, n, x, w["attn_norm"], first)
        L.close(first[:n], *L.rms(x, w["attn_norm"], EPS), self.t)
        L.close(qkv.flatten(1), *L.linear(first[:n], w["qkv"], w["qkv_bias"]), self.t)
        xv, at, qv = qkv.float().cpu().numpy(), 0, np.zeros((n, HQ, D), np.float32)
        weights = [None if w.get(k) is None else w[k].float().cpu().numpy() for k in ("q_norm", "k_norm")]
        norm = head_norm if "q_norm" in w else (lambda v, weight, eps: v)
        for b, m in enumerate(new):
            self.c.lens[b] += m
            ln = int(self.c.lens[b])
            cs, sn, rows = self.cos[ln - m:ln][:, None], self.sin[ln - m:ln][:, None], xv[at:at + m]
            qv[at:at + m] = rope(norm(rows[:, :HQ], weights[0], EPS), cs, sn, False)
            k = rope(norm(rows[:, HQ:HQ + HKV], weights[1], EPS), cs, sn, False)
            append_chunk(self.kind, self.c.k, self.c.ks, self.c.tables[b], ln, k, False)
            append_chunk(self.kind, self.c.v, self.c.vs, self.c.tables[b], ln, rows[:, HQ + HKV:], True)
            at += m
        q = torch.from_numpy(qv).to(L.TYPES[self.t])
        assert torch.equal(y.q[:n].cpu(), q)
        at = 0
        for b, m in enumerate(new):
            want, tol = reference(self.c, b, q[at:at + m].double().numpy())
            close(y.o[at:at + m], want, tol, self.t == "bf16")
            at += m
        # The residual stream between the two blocks is overwritten too: what the output holds without the last product.
        from paper_2509_00195_amd import tts_linear

        mid = torch.empty_like(x)
        tts_linear(y.lin_out, n, y.o[:n].flatten(1), w["out"], mid, None, x, y.ws, y.ws.numel())
        L.close(mid, *L.linear(y.o[:n].flatten(1), w["out"], residual=x), self.t)
        L.close(y.normed[:n], *L.rms(mid, w["ffn_norm"], EPS), self.t)
        L.close(y.ffn[:n], *L.gated(y.normed[:n], w["gate"], w["up"]), self.t)
        L.close(out, *L.linear(y.ffn[:n], w["down"], residual=mid), self.t)


@pytest.mark.parametrize("kind,heads", [(k, True) for k in KINDS] + [("bf16", False)])
def test_prompts_then_decode_steps(kind, heads):
    m = Model(kind, 5, 1, heads)
    for new in ([37, 1, 16, 60, 5], [3, 20, 31, 2, 1]):
        x = m.hidden(sum(new))
        m.lens += _up(np.array(new, np.int32))
        offs = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        m.check(x, m.run(x.clone(), offs), new)
    meta = tts_build_prefix_meta(np.array([0, 5], np.int32), m.c.tables, m.c.lens, BS, m.c.nb, desc=m.desc)
    for step in range(6):
        x = m.hidden(5)
        m.lens += 1
        m.check(x, m.run(x.clone(), meta=meta if step % 2 else None), [1] * 5)


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_captured_step(kind):
    """A chunk and a decode step in one graph, replayed beside eager work: every replay leaves what eager calls leave."""
    m, e = Model(kind, 4, 2), Model(kind, 4, 2)
    new = [9, 1, 30, 4]
    offs = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    bufs = [[torch.zeros((n, HIDDEN), dtype=torch.bfloat16, device=DEV) for n in (sum(new), 4)] for _ in range(2)]

    def step(model, b, stream=None):
        model.run(b[0], offs, stream=stream)
        model.lens += 1
        model.run(b[1], stream=stream)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    m.lens.copy_(torch.tensor([40, 3, 60, 30], dtype=torch.int32, device=DEV))
    step(m, bufs[0])  # allocates what the calls need
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(m, bufs[0], side)
    for t, s in zip(m.dev, e.dev):
        if t is not None:
            t.copy_(s)
    for rep in range(4):
        fresh = [m.hidden(len(b)) for b in bufs[0]]
        for b in bufs:
            for t, s in zip(b, fresh):
                t.copy_(s)
        start = torch.tensor([40 + 5 * rep, 3 + rep, 60, 30 + rep], dtype=torch.int32, device=DEV)
        m.lens.copy_(start)
        e.lens.copy_(start)
        step(e, bufs[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        print(f"{kind} replay {rep}", flush=True)
        assert all(torch.equal(a, b) for a, b in zip(*bufs)), rep
        for a, b in zip(m.dev, e.dev):
            assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), rep
