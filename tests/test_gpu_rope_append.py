"""The rotating append against the oracle, bit for bit: fp32 products and sums rounded one by one leave nothing open."""

import numpy as np
import pytest
import torch

from oracle.cached_ops import append_chunk, rope
from paper_2509_00195_amd import make_rope, tts_append_kv, tts_copy_blocks, tts_rope_append_kv, tts_rope_tables
from tests._cached import BS, DEV, KINDS, Cache, desc_of

pytestmark = pytest.mark.gpu


def _host(t):
    a = t.cpu()
    return a.view(torch.int16).numpy().view(np.uint16) if a.dtype == torch.bfloat16 else a.numpy()


def _up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Batch:
    """Random tokens of a batch in one projection's output, and the cache they go to."""

    def __init__(self, kind, hq, hkv, d, lens, new, rot, inter, seed, pad=0, gap=0, max_pos=None, boost=()):
        rng = np.random.default_rng(seed)
        self.kind, self.hq, self.hkv, self.d, self.rot, self.inter = kind, hq, hkv, d, rot, inter
        self.lens, self.new = np.asarray(lens, np.int32), list(new)
        self.cache = Cache(kind, hkv, d, np.maximum(self.lens, 0), rng)
        self.offs = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.total = int(self.offs[-1])
        wide = torch.float32 if kind == "f32" else torch.bfloat16
        rows = hq + 2 * hkv
        x = torch.from_numpy(rng.standard_normal((self.total + pad, rows * d + gap)).astype(np.float32))
        for b in boost:  # tokens beyond their block's scale
            x[self.offs[b]:self.offs[b + 1]] *= 40
        x = x.to(wide)
        self.flat = x.to(DEV)
        self.qkv = self.flat[:, :rows * d].unflatten(1, (rows, d))
        self.values = x.float().numpy()[:, :rows * d].reshape(-1, rows, d)
        self.max_pos = max_pos or max(1, int(self.lens.max()))
        self.cos, self.sin = tts_rope_tables(rot, 1e4, self.max_pos)
        self.rope = make_rope(_up(self.cos), _up(self.sin), inter)
        self.keep = (_up(self.cos), _up(self.sin))
        self.rope = make_rope(*self.keep, inter)
        self.q_out = torch.full((self.total + pad, hq, d), 7.0, dtype=wide, device=DEV)

    def call(self, num_tokens=None, positions=None, tok_offsets=True, q=True, **kw):
        c, x = self.cache, self.qkv
        self.dev = c.device()
        tts_rope_append_kv(desc_of(self.kind, self.hq, self.hkv, self.d), len(self.lens),
                           x.shape[0] if num_tokens is None else num_tokens, x[:, self.hq:self.hq + self.hkv],
                           x[:, self.hq + self.hkv:], _up(c.tables), c.tables.shape[1], _up(self.lens), c.nb, *self.dev,
                           rope=self.rope, q=x[:, :self.hq] if q else None, q_out=self.q_out if q else None,
                           tok_offsets=_up(self.offs) if tok_offsets else None,
                           positions=None if positions is None else _up(positions), **kw)
        torch.cuda.synchronize()

    def check(self, positions=None):
        """Everything that the call may write, against the oracle; rows and blocks that it may not, unchanged."""
        c, q = self.cache, _host(self.q_out)
        want_q = np.full(self.q_out.shape, 7.0, np.float32)
        for b, n in enumerate(self.new):
            ln, a = int(self.lens[b]), int(self.offs[b])
            if ln <= 0 or n == 0:
                continue
            if ln < n:
                want_q[a:a + n] = np.nan
                continue
            pos = np.arange(ln - n, ln) if positions is None else positions[a:a + n]
            ok = (pos >= 0) & (pos < self.max_pos) | (self.rot == 0)
            at = np.where(ok, pos, 0) % self.max_pos
            x, cs, sn = self.values[a:a + n], self.cos[at][:, None], self.sin[at][:, None]
            want_q[a:a + n] = np.where(ok[:, None, None], rope(x[:, :self.hq], cs, sn, self.inter), np.nan)
            k = rope(x[:, self.hq:self.hq + self.hkv], cs, sn, self.inter)
            append_chunk(self.kind, c.k, c.ks, c.tables[b], ln, k, False, stored=ok)
            append_chunk(self.kind, c.v, c.vs, c.tables[b], ln, x[:, self.hq + self.hkv:], True, stored=ok)
        if self.kind == "f32":
            assert np.array_equal(q, want_q, equal_nan=True)
        else:
            want = torch.from_numpy(want_q).bfloat16().float().numpy()
            assert np.array_equal((q.astype(np.uint32) << 16).view(np.float32), want, equal_nan=True)
        for name, got, ref in zip(("k", "v", "k_scale", "v_scale"), self.dev, (c.k, c.v, c.ks, c.vs)):
            if ref is not None:
                g = _host(got)
                g, ref = (g.view(np.uint32), ref.view(np.uint32)) if ref.dtype == np.float32 else (g, ref)
                g, ref = (g.view(np.uint16), ref) if ref.dtype == np.uint16 else (g, ref)
                assert np.array_equal(g, ref), name


CHUNKS = ([40, 1, 16, 33, 200, 17, 5, 64], [40, 1, 16, 2, 100, 0, 3, 31])  # lengths, new tokens


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,d,rot,inter", [(4, 1, 64, 64, False), (15, 5, 64, 32, True), (12, 2, 128, 128, False),
                                                (6, 3, 128, 48, False), (8, 8, 64, 24, True), (7, 1, 128, 6, True),
                                                (2, 1, 64, 10, False), (16, 16, 128, 128, True)])
def test_chunks(kind, hq, hkv, d, rot, inter):
    b = Batch(kind, hq, hkv, d, *CHUNKS, rot, inter, 1, boost=(3, 6))
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gap", [0, 8, 3])
def test_padded_rows_gaps_idle_and_short_sequences(kind, gap):
    """Rows behind the last sequence are left alone; idle sequences too; one shorter than its chunk has NaN queries.
    gap 3: rows at odd addresses, read one by one."""
    lens, new = [40, 0, 16, 9, -3, 50], [7, 4, 16, 12, 2, 3]
    b = Batch(kind, 14, 2, 64, lens, new, 64, False, 2, pad=9, gap=gap)
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_positions(kind):
    """Positions of the caller's, some outside the tables: NaN queries, and nothing of the token stored."""
    b = Batch(kind, 4, 2, 64, [40, 21, 16], [30, 1, 16], 64, False, 3, max_pos=25)
    pos = np.random.default_rng(4).integers(-2, 27, b.total).astype(np.int32)
    pos[0], pos[5] = 25, -1
    pos[[20, 31]] = 24, 0
    b.call(positions=pos)
    b.check(pos)


@pytest.mark.parametrize("kind", KINDS)
def test_bad_tables(kind):
    """Blocks past the table row and ids outside the pool store nothing; the queries are rotated all the same."""
    b = Batch(kind, 4, 2, 64, [100, 40, 33], [60, 10, 33], 64, True, 5)
    b.cache.tables = b.cache.tables[:, :4].copy()
    b.cache.tables[1, 2], b.cache.tables[2, 1], b.cache.tables[0, 3] = b.cache.nb, -1, 1 << 30
    b.call()
    b.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("seqs", [1, 3, 70])
def test_single_tokens(kind, seqs):
    rng = np.random.default_rng(6)
    lens = rng.integers(1, 90, seqs)
    lens[seqs // 2] = 0 if seqs > 1 else 17
    b = Batch(kind, 28, 4, 128, lens, [1] * seqs, 128, False, 7, boost=range(0, seqs, 3))
    b.call(tok_offsets=False)
    b.check()


@pytest.mark.parametrize("kind", KINDS)
def test_without_rotation_is_the_plain_append(kind):
    """rope NULL and one token per sequence: what tts_append_kv leaves, bit for bit; with rot_dim 0 too."""
    seqs = 12
    lens = np.array([1, 17, 33, 5, 16, 64, 0, 9, 20, 45, 2, 65], np.int32)
    b = Batch(kind, 4, 2, 128, lens, [1] * seqs, 0, False, 8, boost=(3, 8, 9))
    x, c = b.qkv, b.cache
    k, v = x[:, 4:6].contiguous(), x[:, 6:].contiguous()
    want = c.device()
    tts_append_kv(desc_of(kind, 4, 2, 128), seqs, k, v, _up(c.tables), c.tables.shape[1], _up(lens), c.nb, *want)
    for kw in (dict(), dict(rope=b.rope), dict(tok_offsets=_up(b.offs))):
        got = c.device()
        tts_rope_append_kv(desc_of(kind, 4, 2, 128), seqs, seqs, x[:, 4:6], x[:, 6:], _up(c.tables), c.tables.shape[1],
                           _up(lens), c.nb, *got, **kw)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert w is None or torch.equal(g.view(torch.uint8), w.view(torch.uint8))


def test_in_place_and_without_queries():
    b = Batch("bf16", 4, 2, 64, [50, 20], [20, 3], 64, False, 9)
    b.call()
    want = b.q_out.clone()
    c, q = b.cache, b.qkv[:, :4].contiguous()
    dev = c.device()
    tts_rope_append_kv(desc_of("bf16", 4, 2, 64), 2, b.total, b.qkv[:, 4:6], b.qkv[:, 6:], _up(c.tables), c.tables.shape[1],
                       _up(b.lens), c.nb, *dev, rope=b.rope, q=q, q_out=q, tok_offsets=_up(b.offs))
    assert torch.equal(q, want)
    none = c.device()
    tts_rope_append_kv(desc_of("bf16", 4, 2, 64), 2, b.total, b.qkv[:, 4:6], b.qkv[:, 6:], _up(c.tables), c.tables.shape[1],
                       _up(b.lens), c.nb, *none, rope=b.rope, tok_offsets=_up(b.offs))
    assert all(torch.equal(x, y) for x, y in zip(dev[:2], none[:2]))


def test_many_sequences_of_odd_chunks():
    """More sequences than a wave searches in one step, empty ones among them."""
    rng = np.random.default_rng(10)
    new = rng.integers(0, 4, 5000)
    lens = new + rng.integers(0, 20, 5000)
    b = Batch("mx4", 2, 1, 64, lens, new, 64, False, 11)
    b.call()
    b.check()


def test_infinities_and_nan_in_a_4bit_group():
    """A group that holds one reads back as NaN (scale byte 255, codes 0); its neighbours are as without it."""
    b = Batch("mx4", 2, 2, 64, [20], [20], 0, False, 12)
    x = b.values
    for t, h, i, v in ((3, 2, 5, np.inf), (4, 3, 40, np.nan), (9, 4, 1, -np.inf), (9, 5, 63, np.nan)):
        x[t, h, i] = v
        b.qkv[t, h, i] = float(v)
    b.call(q=False)
    c = b.cache
    append_chunk("mx4", c.k, None, c.tables[0], 20, x[:, 2:4], False)
    append_chunk("mx4", c.v, None, c.tables[0], 20, x[:, 4:], True)
    assert np.array_equal(_host(b.dev[0]), c.k) and np.array_equal(_host(b.dev[1]), c.v)
    half = BS * 64 // 2
    assert (c.k[..., half:] == 255).sum() == 2 and (c.v[..., half:] == 255).sum() == 2


@pytest.mark.parametrize("kind", ["bf16", "mx4"])
def test_offsets_past_32_bits(kind):
    """A cache of over 4 GiB per tensor: blocks at its end."""
    hkv, d = 8, 128
    per = hkv * BS * d * 2 if kind == "bf16" else hkv * 17 * d // 2
    nb = (1 << 32) // per + 40
    shape = (nb, per) if kind == "mx4" else (nb, per // 2)
    dt = torch.uint8 if kind == "mx4" else torch.bfloat16
    b = Batch(kind, 8, hkv, d, [33, 20], [33, 1], 128, False, 13)
    c = b.cache
    kd, vd = (torch.empty(shape, dtype=dt, device=DEV) for _ in range(2))
    shift = nb - c.nb
    small = c.device()
    for big, s in ((kd, small[0]), (vd, small[1])):
        big[shift:] = s.reshape(c.nb, -1).view(dt)
    tables = np.where(c.tables >= 0, c.tables + shift, c.tables).astype(np.int32)
    x = b.qkv
    tts_rope_append_kv(desc_of(kind, 8, hkv, d), 2, b.total, x[:, 8:16], x[:, 16:], _up(tables), tables.shape[1], _up(b.lens),
                       nb, kd, vd, rope=b.rope, q=x[:, :8], q_out=b.q_out, tok_offsets=_up(b.offs))
    torch.cuda.synchronize()
    b.dev = tuple(t[shift:].clone().view(s.dtype).reshape(s.shape) for t, s in ((kd, small[0]), (vd, small[1]))) + (None, None)
    b.check()


def test_copies_of_4bit_blocks():
    rng = np.random.default_rng(14)
    c = Cache("mx4", 5, 64, [100], rng, spare=9)
    pairs = np.array([[0, 10], [3, 11], [0, 12], [5, 5], [c.nb, 1], [2, -1]], np.int32)
    k, v, _, _ = c.device()
    tts_copy_blocks(desc_of("mx4", 5, 5, 64), len(pairs), _up(pairs), c.nb, k, v)
    for s, d in ((0, 10), (3, 11), (0, 12)):
        c.k[d], c.v[d] = c.k[s], c.v[s]
    assert np.array_equal(_host(k), c.k) and np.array_equal(_host(v), c.v)
