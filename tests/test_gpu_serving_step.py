"""The operators around cached attention as a program runs them together: chunks appended with their rotation and
attended to, then decode steps (append, paged and prefix-shared attention), eager and captured into a graph."""

import numpy as np
import pytest
import torch

from oracle.cached_ops import append_chunk, rope
from paper_2509_00195_amd import (make_rope, tts_build_prefix_meta, tts_paged_decode_attn, tts_paged_decode_workspace_size,
                                  tts_paged_prefill_attn, tts_paged_prefill_workspace_size, tts_prefix_decode_attn,
                                  tts_prefix_decode_workspace_size, tts_rope_append_kv, tts_rope_tables)
from tests._cached import BS, DEV, KINDS, Cache, close, desc_of, reference

pytestmark = pytest.mark.gpu
HQ, HKV, D, ROOM = 8, 2, 64, 160


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Model:
    """One layer's cached attention over sequences that grow, beside the oracle's cache."""

    def __init__(self, kind, seqs, seed):
        self.rng = np.random.default_rng(seed)
        self.kind, self.seqs = kind, seqs
        self.wide = torch.float32 if kind == "f32" else torch.bfloat16
        self.out_t = "f32" if kind == "f32" else "bf16"
        self.desc = desc_of(kind, HQ, HKV, D, self.out_t)
        self.c = Cache(kind, HKV, D, [ROOM] * seqs, self.rng)
        self.c.lens = np.zeros(seqs, np.int32)
        self.dev = self.c.device()
        self.tables = _up(self.c.tables)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=DEV)
        self.cos, self.sin = tts_rope_tables(D, 1e4, ROOM)
        self.tabs = (_up(self.cos), _up(self.sin))
        self.rope = make_rope(*self.tabs)
        self.cols = self.c.tables.shape[1]

    def tokens(self, n):
        x = torch.from_numpy(self.rng.standard_normal((n, HQ + 2 * HKV, D)).astype(np.float32)).to(self.wide)
        return x.to(DEV), x.float().numpy()

    def append(self, x, q_out, offs=None, stream=None):
        tts_rope_append_kv(self.desc, self.seqs, x.shape[0], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], self.tables, self.cols,
                           self.lens, self.c.nb, *self.dev, rope=self.rope, q=x[:, :HQ], q_out=q_out, tok_offsets=offs,
                           stream=stream)

    def oracle_append(self, xv, new):
        """The oracle's cache after the new tokens, and the rotated queries as values."""
        at, q = 0, np.zeros((len(xv), HQ, D), np.float32)
        for b, n in enumerate(new):
            self.c.lens[b] += n
            ln = int(self.c.lens[b])
            cs, sn = self.cos[ln - n:ln][:, None], self.sin[ln - n:ln][:, None]
            q[at:at + n] = rope(xv[at:at + n, :HQ], cs, sn, False)
            append_chunk(self.kind, self.c.k, self.c.ks, self.c.tables[b], ln, rope(xv[at:at + n, HQ:HQ + HKV], cs, sn, False),
                         False)
            append_chunk(self.kind, self.c.v, self.c.vs, self.c.tables[b], ln, xv[at:at + n, HQ + HKV:], True)
            at += n
        return torch.from_numpy(q).to(self.wide).double().numpy()

    def check(self, out, qv, new):
        at = 0
        for b, n in enumerate(new):
            want, tol = reference(self.c, b, qv[at:at + n])
            close(out[at:at + n], want, tol, self.out_t == "bf16")
            at += n


@pytest.mark.parametrize("kind", KINDS)
def test_prefill_then_decode_steps(kind):
    m = Model(kind, 5, 1)
    for new in ([37, 1, 16, 60, 5], [3, 20, 31, 2, 1]):  # two chunks of each sequence
        x, xv = m.tokens(sum(new))
        qv = m.oracle_append(xv, new)
        m.lens.copy_(_up(m.c.lens))
        offs = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        q, out = (torch.zeros((sum(new), HQ, D), dtype=m.wide, device=DEV) for _ in range(2))
        m.append(x, q, offs)
        size = tts_paged_prefill_workspace_size(m.desc, m.seqs, sum(new), ROOM)
        ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
        tts_paged_prefill_attn(m.desc, m.seqs, sum(new), offs, q, *m.dev, m.tables, m.cols, m.lens, ROOM, m.c.nb, out, ws, size)
        assert np.array_equal(q.double().cpu().numpy(), qv)
        m.check(out, qv, new)
    meta = tts_build_prefix_meta(np.array([0, m.seqs], np.int32), m.c.tables, m.c.lens, BS, m.c.nb, desc=m.desc)
    size = max(tts_paged_decode_workspace_size(m.desc, m.seqs, ROOM), tts_prefix_decode_workspace_size(m.desc, meta))
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    new = [1] * m.seqs
    for step in range(20):
        x, xv = m.tokens(m.seqs)
        qv = m.oracle_append(xv, new)
        m.lens += 1
        q, out, shared = (torch.zeros((m.seqs, HQ, D), dtype=m.wide, device=DEV) for _ in range(3))
        m.append(x, q)
        tts_paged_decode_attn(m.desc, m.seqs, q, *m.dev, m.tables, m.cols, m.lens, ROOM, m.c.nb, out, ws, size)
        if step % 5 == 4:
            torch.cuda.synchronize()
            m.check(out, qv, new)
            tts_prefix_decode_attn(m.desc, meta, q, *m.dev, m.tables, m.cols, m.lens, m.c.nb, shared, ws, size)
            m.check(shared, qv, new)


@pytest.mark.parametrize("kind", KINDS)
def test_captured_step(kind):
    """A decode step and a chunk's append and attention in one graph, replayed beside eager work: every replay leaves
    what the eager calls leave."""
    m, e = Model(kind, 4, 2), Model(kind, 4, 2)
    new = [9, 1, 30, 4]
    offs = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    total = sum(new)
    sizes = [tts_paged_prefill_workspace_size(m.desc, 4, total, ROOM), tts_paged_decode_workspace_size(m.desc, 4, ROOM)]
    ws = [torch.empty(max(s, 1), dtype=torch.uint8, device=DEV) for s in sizes]
    x, _ = m.tokens(total)
    x1, _ = m.tokens(4)
    bufs = {k: [torch.zeros((n, HQ, D), dtype=m.wide, device=DEV) for n in (total, total, 4, 4)] for k in "me"}

    def step(model, b, x, x1, stream=None):
        model.append(x, b[0], offs, stream)
        tts_paged_prefill_attn(model.desc, 4, total, offs, b[0], *model.dev, model.tables, model.cols, model.lens, ROOM,
                               model.c.nb, b[1], ws[0], sizes[0], stream)
        model.lens += 1
        model.append(x1, b[2], None, stream)
        tts_paged_decode_attn(model.desc, 4, b[2], *model.dev, model.tables, model.cols, model.lens, ROOM, model.c.nb, b[3],
                              ws[1], sizes[1], stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(m, bufs["m"], x, x1, side)
    torch.cuda.synchronize()
    for rep in range(4):
        fresh, _ = m.tokens(total)
        fresh1, _ = m.tokens(4)
        x.copy_(fresh)
        x1.copy_(fresh1)
        start = torch.tensor([40 + 5 * rep, 3 + rep, 60, 30 + rep], dtype=torch.int32, device=DEV)
        m.lens.copy_(start)
        e.lens.copy_(start)
        step(e, bufs["e"], x, x1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        print(f"{kind} replay {rep}", flush=True)
        for a, b in zip(bufs["m"], bufs["e"]):
            assert torch.equal(a, b), rep
        for a, b in zip(m.dev, e.dev):
            assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), rep


def test_two_streams():
    """Calls of two models on two streams at once, each with its own workspace: as one after the other."""
    models = [Model("mx4", 3, 3), Model("bf16", 3, 4)]
    streams = [torch.cuda.Stream() for _ in models]
    new = [50, 7, 90]
    offs = _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    xs = [m.tokens(sum(new))[0] for m in models]
    outs = []
    for m in models:
        m.lens.copy_(torch.tensor([60, 70, 95], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for together in (False, True):
        res = []
        for m, s, x in zip(models, streams, xs):
            q, out = (torch.zeros((sum(new), HQ, D), dtype=m.wide, device=DEV) for _ in range(2))
            torch.cuda.synchronize()
            res.append((m, s, x, q, out))
        for _ in range(3):
            for m, s, x, q, out in res:
                m.append(x, q, offs, s)
                tts_paged_prefill_attn(m.desc, m.seqs, sum(new), offs, q, *m.dev, m.tables, m.cols, m.lens, ROOM, m.c.nb, out,
                                       None, 0, s)
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        outs.append([(q, out) for _, _, _, q, out in res])
    for (q0, o0), (q1, o1) in zip(*outs):
        assert torch.equal(q0, q1) and torch.equal(o0, o1)
