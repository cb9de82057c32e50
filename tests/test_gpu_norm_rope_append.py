"""The append with head norms against the oracle, bit for bit: mean and root in 64 bits, then products rounded one by one."""

import numpy as np
import pytest
import torch

from oracle.cached_ops import append_chunk, rope
from oracle.layer_ops import head_norm
from paper_2509_00195_amd import make_head_norm, tts_norm_rope_append_kv, tts_rope_append_kv
from tests._cached import DEV, KINDS, desc_of
from tests.test_gpu_rope_append import CHUNKS, Batch, _host, _up

pytestmark = pytest.mark.gpu


class NormBatch(Batch):
    def __init__(self, *args, weights=True, eps=1e-6, shift=0, **kw):
        super().__init__(*args, **kw)
        rng = np.random.default_rng(99)
        wide = self.flat.dtype
        self.eps, self.w = eps, [None, None]
        self.dev_w = [None, None]
        if weights:
            for i in range(2):
                t = torch.from_numpy((1 + 0.3 * rng.standard_normal(self.d + shift)).astype(np.float32)).to(wide)[shift:]
                self.w[i] = t.float().numpy()
                self.dev_w[i] = torch.empty(self.d + shift, dtype=wide, device=DEV)[shift:].copy_(t)
        self.norm = make_head_norm(*self.dev_w, eps)

    def call(self, num_tokens=None, positions=None, tok_offsets=True, q=True, rope=True, **kw):
        c, x = self.cache, self.qkv
        self.dev = c.device()
        tts_norm_rope_append_kv(desc_of(self.kind, self.hq, self.hkv, self.d), self.norm, len(self.lens),
                                x.shape[0] if num_tokens is None else num_tokens, x[:, self.hq:self.hq + self.hkv],
                                x[:, self.hq + self.hkv:], _up(c.tables), c.tables.shape[1], _up(self.lens), c.nb, *self.dev,
                                rope=self.rope if rope else None, q=x[:, :self.hq] if q else None,
                                q_out=self.q_out if q else None, tok_offsets=_up(self.offs) if tok_offsets else None,
                                positions=None if positions is None else _up(positions), **kw)
        torch.cuda.synchronize()

    def check(self, positions=None):
        """As the append without norms, of heads that the oracle has normalised."""
        hq, hkv = self.hq, self.hkv
        self.values = self.values.copy()
        self.values[:, :hq] = head_norm(self.values[:, :hq], self.w[0], self.eps)
        self.values[:, hq:hq + hkv] = head_norm(self.values[:, hq:hq + hkv], self.w[1], self.eps)
        super().check(positions)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,d,rot,inter", [(4, 1, 64, 64, False), (15, 5, 64, 32, True), (12, 2, 128, 128, False),
                                                (6, 3, 128, 48, False), (8, 8, 64, 24, True), (7, 1, 128, 6, True),
                                                (2, 1, 64, 10, False), (16, 16, 128, 128, True), (28, 4, 128, 64, False),
                                                (5, 1, 128, 2, False), (9, 3, 64, 0, False)])
def test_chunks(kind, hq, hkv, d, rot, inter):
    """Rotations whose units fill their lanes, and ones that leave some idle or take two each."""
    b = NormBatch(kind, hq, hkv, d, *CHUNKS, rot, inter, 1, boost=(3, 6))
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gap,shift", [(0, 0), (8, 1), (3, 0)])
def test_padded_rows_gaps_idle_and_short_sequences(kind, gap, shift):
    """gap 3: rows at odd addresses; shift 1: weights at one."""
    lens, new = [40, 0, 16, 9, -3, 50], [7, 4, 16, 12, 2, 3]
    b = NormBatch(kind, 14, 2, 64, lens, new, 64, False, 2, pad=9, gap=gap, shift=shift)
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_positions(kind):
    b = NormBatch(kind, 4, 2, 64, [40, 21, 16], [30, 1, 16], 64, False, 3, max_pos=25)
    pos = np.random.default_rng(4).integers(-2, 27, b.total).astype(np.int32)
    pos[0], pos[5] = 25, -1
    pos[[20, 31]] = 24, 0
    b.call(positions=pos)
    b.check(pos)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("seqs", [1, 3, 70])
def test_single_tokens(kind, seqs):
    rng = np.random.default_rng(6)
    lens = rng.integers(1, 90, seqs)
    lens[seqs // 2] = 0 if seqs > 1 else 17
    b = NormBatch(kind, 28, 4, 128, lens, [1] * seqs, 128, False, 7, boost=range(0, seqs, 3))
    b.call(tok_offsets=False)
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("weights,eps", [(False, 0.25), (True, 0.0)])
def test_without_weights_and_without_a_rotation(kind, weights, eps):
    b = NormBatch(kind, 6, 2, 64, [30, 9], [21, 9], 0, False, 8, weights=weights, eps=eps)
    b.call(rope=False)
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_bad_tables(kind):
    b = NormBatch(kind, 4, 2, 64, [100, 40, 33], [60, 10, 33], 64, True, 5)
    b.cache.tables = b.cache.tables[:, :4].copy()
    b.cache.tables[1, 2], b.cache.tables[2, 1], b.cache.tables[0, 3] = b.cache.nb, -1, 1 << 30
    b.call()
    b.check()


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (24, False)])
@pytest.mark.parametrize("shift", [0, 1])
def test_in_place_and_without_queries(rot, inter, shift):
    b = NormBatch("bf16", 4, 2, 64, [50, 20], [20, 3], rot, inter, 9)
    b.call()
    want = b.q_out.clone()
    c = b.cache
    q = torch.empty(b.total * 4 * 64 + shift, dtype=torch.bfloat16, device=DEV)[shift:].view(b.total, 4, 64).copy_(b.qkv[:, :4])
    dev = c.device()
    args = (b.norm, 2, b.total, b.qkv[:, 4:6], b.qkv[:, 6:], _up(c.tables), c.tables.shape[1], _up(b.lens), c.nb)
    tts_norm_rope_append_kv(desc_of("bf16", 4, 2, 64), *args, *dev, rope=b.rope, q=q, q_out=q, tok_offsets=_up(b.offs))
    assert torch.equal(q, want)
    none = c.device()
    tts_norm_rope_append_kv(desc_of("bf16", 4, 2, 64), *args, *none, rope=b.rope, tok_offsets=_up(b.offs))
    assert all(torch.equal(x, y) for x, y in zip(dev[:2], none[:2]))


def test_heads_that_are_not_finite_and_zeros():
    """An infinity leaves its head's other elements 0 and is NaN itself, a NaN makes the head NaN, zeros stay zeros; the
    other heads are as without them."""
    b = NormBatch("f32", 3, 1, 64, [9], [9], 0, False, 12)
    x = b.values
    for t, h, i, v in ((2, 0, 5, np.inf), (3, 1, 7, np.nan), (4, 3, 9, -np.inf), (5, 3, 0, np.nan)):
        x[t, h, i] = v
        b.qkv[t, h, i] = float(v)
    x[6], b.qkv[6] = 0, 0
    b.call()
    with np.errstate(invalid="ignore"):
        q = head_norm(x[:, :3], b.w[0], b.eps)
        k = head_norm(x[:, 3:4], b.w[1], b.eps)
    assert np.array_equal(_host(b.q_out), q, equal_nan=True)
    assert np.isnan(q[2, 0, 5]) and (q[2, 0, :5] == 0).all() and np.isnan(q[3, 1]).all() and (q[6] == 0).all()
    append_chunk("f32", b.cache.k, None, b.cache.tables[0], 9, k, False)
    assert np.array_equal(_host(b.dev[0]), b.cache.k, equal_nan=True)


def test_values_are_stored_as_without_norms():
    b = NormBatch("fp8", 8, 2, 128, [40, 3], [20, 3], 128, False, 13)
    b.call()
    c, dev = b.cache, b.cache.device()
    tts_rope_append_kv(desc_of("fp8", 8, 2, 128), 2, b.total, b.qkv[:, 8:10], b.qkv[:, 10:], _up(c.tables),
                       c.tables.shape[1], _up(b.lens), c.nb, *dev, rope=b.rope, tok_offsets=_up(b.offs))
    assert torch.equal(b.dev[1], dev[1]) and torch.equal(b.dev[3], dev[3])
    assert not torch.equal(b.dev[0], dev[0])


def test_many_sequences_of_odd_chunks():
    rng = np.random.default_rng(10)
    new = rng.integers(0, 4, 5000)
    b = NormBatch("mx4", 2, 1, 64, new + rng.integers(0, 20, 5000), new, 64, False, 11)
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_captured_and_replayed(kind):
    b = NormBatch(kind, 12, 2, 128, *CHUNKS, 128, False, 14)
    c, x = b.cache, b.qkv
    up = [_up(a) for a in (c.tables, b.lens, b.offs)]
    start = c.device()
    dev, other = ([None if t is None else t.clone() for t in start] for _ in range(2))
    q_other = torch.empty_like(b.q_out)

    def call(dev, q_out, stream=None):
        tts_norm_rope_append_kv(desc_of(kind, 12, 2, 128), b.norm, len(b.lens), b.total, x[:, 12:14], x[:, 14:], up[0],
                                c.tables.shape[1], up[1], c.nb, *dev, rope=b.rope, q=x[:, :12], q_out=q_out,
                                tok_offsets=up[2], stream=stream)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(dev, b.q_out, side)
    for rep in range(4):
        x.copy_(torch.randn(x.shape, device=DEV))
        for t in (dev, other):
            for a, s in zip(t, start):
                if a is not None:
                    a.copy_(s)
        call(other, q_other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.q_out, q_other), rep
        for a, e in zip(dev, other):
            assert a is None or torch.equal(a.view(torch.uint8), e.view(torch.uint8)), rep


def test_rope_is_the_same_without_norms():
    """Rows whose mean square is 1 - eps to the last bit keep their values under the norm: the two calls agree."""
    b = NormBatch("f32", 4, 2, 64, [25, 7], [25, 7], 64, False, 15, weights=False, eps=0.25)
    rng = np.random.default_rng(16)
    signs = np.where(rng.random(b.values.shape) < 0.5, -1.0, 1.0).astype(np.float32)
    half = np.zeros(64, np.float32)
    half[rng.permutation(64)[:48]] = 1.0  # 48 of 64 ones: mean square 0.75
    x = signs * half
    b.values[:] = x
    b.qkv.copy_(torch.from_numpy(x))
    b.call()
    q, k = b.q_out.clone(), b.dev[0].clone()
    Batch.call(b)
    assert torch.equal(q, b.q_out) and torch.equal(k, b.dev[0])
    cs, sn = b.cos[:25][:, None], b.sin[:25][:, None]
    assert np.array_equal(_host(q[:25]), rope(x[:25, :4], cs, sn, False))
