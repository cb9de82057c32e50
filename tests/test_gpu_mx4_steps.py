"""4-bit caches in the steps of a search: a verification step (append, verification attention) and a decode step (append,
prefix-shared attention), eager, captured and replayed; and a re-plan after a fork."""

import numpy as np
import pytest
import torch

from oracle.cached_ops import append_chunk, rope
from paper_2509_00195_amd import (make_rope, tts_build_prefix_meta, tts_build_verify_meta, tts_fork_prefix_meta,
                                  tts_prefix_decode_attn, tts_prefix_decode_workspace_size, tts_prefix_verify_attn,
                                  tts_rope_append_kv, tts_rope_tables)
from tests._cached import BS, DEV, Cache, close, desc_of, queries, reference

pytestmark = pytest.mark.gpu
HQ, HKV, D, BEAMS, SHARE = 8, 2, 64, 24, 9


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _tree(seed):
    """Two requests of twelve beams; each request's share nine blocks."""
    rng = np.random.default_rng(seed)
    c = Cache("mx4", HKV, D, 16 * SHARE + rng.integers(4, 60, BEAMS), rng)
    for r in (0, 12):
        c.tables[r:r + 12, :SHARE] = c.tables[r, :SHARE]
    return c, np.array([0, 12, BEAMS], np.int32)


class Step:
    """n new tokens of every beam: appended with their rotation, and attended to."""

    def __init__(self, c, offs, n):
        self.n, self.desc = n, desc_of("mx4", HQ, HKV, D, "bf16")
        build = (c.tables, c.lens, n, BS, c.nb) if n > 1 else (c.tables, c.lens, BS, c.nb)
        self.meta = (tts_build_verify_meta if n > 1 else tts_build_prefix_meta)(offs, *build, desc=self.desc)
        self.size = tts_prefix_decode_workspace_size(self.desc, self.meta)
        self.ws = torch.empty(self.size, dtype=torch.uint8, device=DEV)
        self.k, self.v, _, _ = c.device()
        self.tables, self.lens, self.nb = _up(c.tables), _up(c.lens), c.nb
        self.cos, self.sin = tts_rope_tables(D, 1e4, 300)
        self.tabs = (_up(self.cos), _up(self.sin))
        self.rope = make_rope(*self.tabs)
        self.offs = _up(np.arange(0, n * BEAMS + 1, n, dtype=np.int32)) if n > 1 else None
        self.q, self.out = (torch.zeros((n * BEAMS, HQ, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def __call__(self, x, stream=None):
        cols, total = self.tables.shape[1], self.n * BEAMS
        tts_rope_append_kv(self.desc, BEAMS, total, x[:, HQ:HQ + HKV], x[:, HQ + HKV:], self.tables, cols, self.lens, self.nb,
                           self.k, self.v, rope=self.rope, q=x[:, :HQ], q_out=self.q, tok_offsets=self.offs, stream=stream)
        call = tts_prefix_verify_attn if self.n > 1 else tts_prefix_decode_attn
        call(self.desc, self.meta, self.q, self.k, self.v, None, None, self.tables, cols, self.lens, self.nb, self.out, self.ws,
             self.size, stream)

    def check(self, c, xv):
        """Against the oracle, whose cache takes the tokens too."""
        n = self.n
        for b in range(BEAMS):
            ln, row = int(c.lens[b]), xv[n * b:n * b + n]
            cs, sn = self.cos[ln - n:ln][:, None], self.sin[ln - n:ln][:, None]
            append_chunk("mx4", c.k, None, c.tables[b], ln, rope(row[:, HQ:HQ + HKV], cs, sn, False), False)
            append_chunk("mx4", c.v, None, c.tables[b], ln, row[:, HQ + HKV:], True)
        assert np.array_equal(self.k.cpu().numpy(), c.k) and np.array_equal(self.v.cpu().numpy(), c.v)
        q = self.q.double().cpu().numpy()
        for b in range(BEAMS):
            want, tol = reference(c, b, q[n * b:n * b + n])
            close(self.out[n * b:n * b + n], want, tol, True)


def _tokens(rng, n):
    x = torch.from_numpy(rng.standard_normal((n * BEAMS, HQ + 2 * HKV, D)).astype(np.float32)).bfloat16()
    return x.to(DEV), x.float().numpy()


@pytest.mark.parametrize("n", [1, 3])
def test_step_and_its_graph(n):
    rng = np.random.default_rng(1)
    c, offs = _tree(0)
    eager, other = Step(c, offs, n), Step(c, offs, n)
    x, xv = _tokens(rng, n)
    eager(x)
    torch.cuda.synchronize()
    eager.check(c, xv)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        other(x, side)
    torch.cuda.synchronize()
    for rep in range(4):
        x.copy_(_tokens(rng, n)[0])
        eager(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((eager.out, other.out), (eager.q, other.q), (eager.k, other.k), (eager.v, other.v)):
            assert torch.equal(a, b), rep


@pytest.mark.parametrize("beams", [24, 96])
def test_replan_after_a_fork(beams):
    """Half of the beams replaced by copies of others, which share all of their whole blocks."""
    rng = np.random.default_rng(2)
    c = Cache("mx4", HKV, D, 16 * SHARE + rng.integers(4, 200, beams), rng)
    c.tables[:, :SHARE] = c.tables[0, :SHARE]
    offs = np.array([0, beams], np.int32)
    desc = desc_of("mx4", HQ, HKV, D)
    meta = tts_build_prefix_meta(offs, c.tables, c.lens, BS, c.nb, desc=desc)
    for a in range(0, beams, 2):
        c.tables[a + 1], c.lens[a + 1] = c.tables[a], c.lens[a] // BS * BS
    warm = tts_fork_prefix_meta(meta, offs, c.tables, c.lens, BS, c.nb)
    size = tts_prefix_decode_workspace_size(desc, warm)
    q, qv = queries("mx4", (beams, HQ, D), rng)
    out = torch.zeros((beams, HQ, D), device=DEV)
    tts_prefix_decode_attn(desc, warm, q, *c.device(), _up(c.tables), c.tables.shape[1], _up(c.lens), c.nb, out,
                           torch.empty(size, dtype=torch.uint8, device=DEV), size)
    for b in range(beams):
        want, tol = reference(c, b, qv[b][None])
        close(out[b][None], want, tol)
