"""Performance cases of the operators around a model's cached attention.

* ``rope``: the new tokens of a batch (one per sequence in a decode step, a chunk of each in a prefill) have their
  queries and keys rotated by position, and their keys and values stored in the paged cache.
* ``paged``, ``prefix``, ``verify``: attention over a microscaled 4-bit cache: one token per sequence over its own
  blocks, one per beam over blocks shared along the beams' common prefixes, and several per beam.
* ``prefill``: causal attention of a ragged chunk of each sequence's last tokens over its paged cache.

A case is a dict: the attention shape (``hq``, ``hkv``, ``d``) and the type of the cache (``dtype``: f32, bf16, fp8
with a scale per block, mx4 with a scale per 32 head dimensions); ``seqs`` sequences, of which each holds between
``ctx_lo`` and ``ctx_hi`` tokens before the ``q_lo`` to ``q_hi`` new ones; ``rot`` rotated dimensions (``inter``:
neighbouring pairs); ``beams`` to a request and ``share`` tokens of prompt for the prefix-shared calls; ``gain``, the
spread of the attention scores; ``shape``, the number of the lengths drawn.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 16
GROUP = 32  # head dimensions to a microscale
DEVICE = "cuda:0"
FP8_MAX = 448.0
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

_SMALL = dict(hq=12, hkv=2, d=128)
_LARGE = dict(hq=28, hkv=4, d=128)
_ODD = dict(hq=15, hkv=5, d=64)
_BASE = dict(dtype="bf16", seqs=1, ctx_lo=0, ctx_hi=0, q_lo=1, q_hi=1, rot=128, inter=False, beams=1, share=0, gain=1.0,
             shape=0)


def _case(name, kind, heads, **kw):
    return {"name": name, "kind": kind, **_BASE, **heads, **kw}


def listed():
    return [
        # The smallest call: a decode step's tokens of a 1.5B-shaped generator with 16 beams. Latency counts.
        _case("rope_decode_1p5b16", "rope", _SMALL, seqs=16, ctx_lo=512, ctx_hi=2048),
        # The decode step of sixteen requests of 32 beams, 7B-shaped, into an fp8 cache whose scales may grow.
        _case("rope_decode_512_fp8", "rope", _LARGE, dtype="fp8", seqs=512, ctx_lo=64, ctx_hi=700),
        # Prompts and chunks of eight sequences into a 4-bit cache.
        _case("rope_chunks_mx4", "rope", _LARGE, dtype="mx4", seqs=8, q_lo=256, q_hi=2048, ctx_lo=0, ctx_hi=1024),
        # Short ragged chunks, three heads to a cache head, 64-wide heads of which half is rotated in pairs.
        _case("rope_ragged_odd", "rope", _ODD, seqs=11, q_lo=1, q_hi=300, ctx_lo=0, ctx_hi=500, rot=32, inter=True),
        # A 7B-shaped batch of 64 sequences that share nothing.
        _case("mx4_paged_64", "paged", _LARGE, dtype="mx4", seqs=64, ctx_lo=1024, ctx_hi=4095),
        # Few sequences of very long chains of thought: the work is split over the length and joined.
        _case("mx4_paged_long", "paged", _LARGE, dtype="mx4", seqs=4, ctx_lo=60000, ctx_hi=120000),
        # The headline search batch over a 4-bit cache: 64 beams that share a prompt of 1024 tokens.
        _case("mx4_prefix_64", "prefix", _LARGE, dtype="mx4", seqs=64, beams=64, share=1024, ctx_lo=1200, ctx_hi=4000),
        # Verification of three tokens per beam, five requests of eleven beams, 64-wide heads.
        _case("mx4_verify_odd", "verify", _ODD, dtype="mx4", seqs=55, beams=11, share=300, ctx_lo=310, ctx_hi=1500,
              q_lo=3, q_hi=3, gain=2.0),
        # The smallest prefill: one short chunk after a cached prompt.
        _case("prefill_small", "prefill", _SMALL, q_lo=33, q_hi=33, ctx_lo=500, ctx_hi=500),
        # Eight problems' prompts and reasoning steps go to the verifier at once.
        _case("prefill_ragged_8", "prefill", _LARGE, seqs=8, q_lo=200, q_hi=2048),
        # The longest prompt of the framework's own workloads.
        _case("prefill_16k", "prefill", _LARGE, q_lo=16384, q_hi=16384),
        # Chunks that extend long chains of thought in an fp8 cache: few rows over many tokens.
        _case("prefill_chunks_fp8", "prefill", _LARGE, dtype="fp8", seqs=4, q_lo=64, q_hi=300, ctx_lo=8000, ctx_hi=16000),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choices(["rope", "paged", "prefix", "verify", "prefill"], [30, 18, 12, 8, 32])[0]
    hq, hkv, d = rng.choice([(4, 1, 64), (14, 2, 64), (15, 5, 64), (12, 2, 128), (28, 4, 128), (28, 4, 128), (16, 2, 128),
                             (32, 8, 128), (40, 8, 128)])
    c = dict(_BASE, kind=kind, hq=hq, hkv=hkv, d=d, rot=d, dtype="mx4", gain=rng.choice([1.0, 2.0, 3.0]),
             shape=rng.randint(0, 1 << 20))
    if kind in ("rope", "prefill"):
        c["dtype"] = rng.choices(["bf16", "fp8", "mx4", "f32"], [40, 20, 30, 10])[0]
    if kind == "rope":
        if rng.random() < 0.4:
            c["rot"] = rng.choice([d // 4, d // 2, 3 * d // 8])
        c["inter"] = rng.random() < 0.4
        if rng.random() < 0.5:
            c.update(seqs=log(1, 512), ctx_hi=log(8, 1500))
        else:
            c.update(seqs=log(1, 32), ctx_hi=log(8, 2000), q_hi=log(4, 4096))
            c["q_hi"] = min(c["q_hi"], max(1, 12000 // c["seqs"]))
            c["q_lo"] = rng.randint(1, c["q_hi"])
        c["ctx_lo"] = rng.randint(0, c["ctx_hi"])
    elif kind == "paged":
        c["seqs"] = log(1, 256)
        c["ctx_hi"] = min(log(16, 120000), 300000 // c["seqs"])
        c["ctx_lo"] = rng.randint(0, c["ctx_hi"])
    elif kind in ("prefix", "verify"):
        c["beams"] = log(2, 64)
        c["seqs"] = c["beams"] * min(log(1, 16), max(1, 128 // c["beams"]))
        c["share"] = log(16, 2048)
        c["ctx_hi"] = c["share"] + log(16, 2000)
        c["ctx_lo"] = rng.randint(c["share"], c["ctx_hi"])
        if kind == "verify":
            c["q_lo"] = c["q_hi"] = rng.randint(2, 8)
            c["beams"] = min(c["beams"], 16)
            c["seqs"] = c["beams"] * max(1, min(c["seqs"], 64) // c["beams"])
    else:
        c["seqs"] = log(1, 16)
        c["q_hi"] = log(2, 8192)
        c["q_lo"] = rng.randint(max(1, c["q_hi"] // 4), c["q_hi"])
        c["ctx_hi"] = log(1, 16000) if rng.random() < 0.6 else 0
        c["ctx_lo"] = rng.randint(c["ctx_hi"] // 2, c["ctx_hi"])
        # No more scores than the longest prompt has.
        while c["seqs"] * c["q_hi"] * (c["ctx_hi"] + c["q_hi"]) * hq > 2e9:
            c["seqs"] = max(1, c["seqs"] // 2)
            c["q_hi"], c["ctx_hi"] = max(2, int(c["q_hi"] * 0.8)), int(c["ctx_hi"] * 0.8)
            c["q_lo"], c["ctx_lo"] = min(c["q_lo"], c["q_hi"]), min(c["ctx_lo"], c["ctx_hi"])
    return c


# ---- lengths and block tables ---------------------------------------------------------------


def _lengths(c):
    """(new tokens, cached tokens with the new ones) of each sequence."""
    rng = np.random.default_rng([c["shape"], 0x5EA])
    new = rng.integers(c["q_lo"], c["q_hi"] + 1, c["seqs"])
    return new.astype(np.int32), (new + rng.integers(c["ctx_lo"], c["ctx_hi"] + 1, c["seqs"])).astype(np.int32)


def _shared_blocks(c, lens):
    """Leading blocks that a beam shares with its whole request, and (half as many more) with its group of four."""
    full = (lens - c["q_hi"]) // BLOCK
    first = np.minimum(c["share"] // BLOCK, full)
    return np.full(len(lens), first.min()), np.minimum(first.min() + c["share"] // BLOCK // 2, full)


def _tables(c, lens, seed):
    """Block tables in a shuffled pool with a tenth of its blocks unused; the pool's size."""
    rng = np.random.default_rng([seed, 0xB10C])
    need = -(-lens.astype(np.int64) // BLOCK)
    cols = np.arange(int(need.max(initial=1)) + 1)
    b = np.arange(len(lens))[:, None]
    name = b * len(cols) + cols[None]  # a block's owner: the beam, its group of four, or its request
    if c["kind"] in ("prefix", "verify"):
        one, four = _shared_blocks(c, lens)
        group = b // c["beams"] * c["beams"] + b % c["beams"] // 4 * 4
        least = np.array([four[(group[:, 0] == g) & (b[:, 0] // c["beams"] == g // c["beams"])].min() for g in group[:, 0]])
        name = np.where(cols[None] < least[:, None], group * len(cols) + cols[None], name)
        name = np.where(cols[None] < one[:, None], b // c["beams"] * c["beams"] * len(cols) + cols[None], name)
    used = cols[None] < need[:, None]
    ids, at = np.unique(name[used], return_inverse=True)
    pool = int(len(ids) * 1.1) + 2
    tables = np.full(name.shape, -1, np.int32)
    tables[used] = rng.permutation(pool)[: len(ids)][at]
    return tables, pool, len(ids)


# ---- inputs -------------------------------------------------------------------------------------


def _power(byte):
    """2 ** (byte - 127) for 1 <= byte <= 254."""
    return (byte.int() << 23).view(torch.float32)


def _mx4(x):
    """Codes (0 .. 15) and scale bytes of the last dimension's groups of 32: the scale is 2 to the exponent of the
    group's largest magnitude less 2; the codes round to the nearest E2M1 value, ties to even, at most 6."""
    y = x.unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1)
    scale = ((top.contiguous().view(torch.int32) >> 23) - 2).clamp_(min=1)  # the exponent's bits, less 2
    m = y * _power(254 - scale)[..., None]
    a = m.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return (code + 8 * torch.signbit(m)).to(torch.uint8).flatten(-2), scale.to(torch.uint8)


def _mx4_pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _mx4_unpack(x):
    return torch.stack([x & 15, x >> 4], -1).flatten(-2)


def _mx4_store(codes, scale, values):
    """A cache of whole blocks from codes [n][heads][16][d] and scales [n][heads][16][d / 32]. Keys: a token's codes
    in a row; values: a dimension's; the block's scales behind them, in the same order."""
    if values:
        codes, scale = codes.transpose(-1, -2), scale.transpose(-1, -2)
    return torch.cat([_mx4_pack(codes).flatten(-2), scale.flatten(-2)], -1).contiguous()


def _mx4_split(x, d, values):
    """Codes [..][16][d] and scale bytes [..][16][d / 32] of blocks as they are stored."""
    codes, scale = _mx4_unpack(x[..., : BLOCK * d // 2]), x[..., BLOCK * d // 2:]
    if values:
        return codes.unflatten(-1, (d, BLOCK)).transpose(-1, -2), scale.unflatten(-1, (d // GROUP, BLOCK)).transpose(-1, -2)
    return codes.unflatten(-1, (BLOCK, d)), scale.unflatten(-1, (BLOCK, d // GROUP))


def _cache(c, pool, gen, values):
    """A cache [pool][hkv][..] of random tokens: channels of unequal spread, as trained keys have. (cache, scales)"""
    hkv, d = c["hkv"], c["d"]
    spread = torch.exp(0.3 * torch.randn((1, hkv, 1, d), generator=gen, device=DEVICE))
    step = max(1, (1 << 27) // (hkv * BLOCK * d))
    parts, scales = [], []
    for a in range(0, pool, step):
        n = min(step, pool - a)
        x = torch.randn((n, hkv, BLOCK, d), generator=gen, device=DEVICE) * spread
        if c["dtype"] == "mx4":
            parts.append(_mx4_store(*_mx4(x), values))
            continue
        x = x.transpose(-1, -2).contiguous() if values else x
        if c["dtype"] == "fp8":
            s = x.abs().flatten(1).amax(1) / FP8_MAX
            scales.append(s)
            x = (x / s.view(-1, 1, 1, 1)).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        parts.append(x if c["dtype"] in ("f32", "fp8") else x.bfloat16())
    return torch.cat(parts), torch.cat(scales) if scales else None


def _inputs(c, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 1000003 + 29)
    new, lens = _lengths(c)
    tables, pool, _ = _tables(c, lens, seed)
    wide = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    offs = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    total, hq, hkv, d = int(offs[-1]), c["hq"], c["hkv"], c["d"]
    s = {"c": c, "pool": pool, "total": total, "tables_h": tables, "lens_h": lens, "max_new": int(new.max()),
         "max_len": int(lens.max()), "tables": torch.from_numpy(tables).to(DEVICE),
         "lens": torch.from_numpy(lens).to(DEVICE), "offs": torch.from_numpy(offs).to(DEVICE)}
    s["k"], s["ks"] = _cache(c, pool, gen, False)
    s["v"], s["vs"] = _cache(c, pool, gen, True)
    if c["kind"] == "rope":
        # One projection's output holds a token's queries, keys and values side by side.
        s["qkv"] = torch.randn((total, hq + 2 * hkv, d), generator=gen, device=DEVICE).to(wide)
        s["q_out"] = torch.zeros((total, hq, d), dtype=wide, device=DEVICE)
        half = c["rot"] // 2
        inv = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=DEVICE) / half)
        angle = torch.arange(s["max_len"], dtype=torch.float64, device=DEVICE)[:, None] * inv
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        # The blocks that the new tokens go to (the program that allotted them knows which).
        row = np.repeat(np.arange(len(new)), -(-lens // BLOCK) - (lens - new) // BLOCK)
        first = np.concatenate([np.arange(a // BLOCK, -(-b // BLOCK)) for a, b in zip(lens - new, lens)])
        s["touched"] = torch.from_numpy(tables[row, first].astype(np.int64)).to(DEVICE)
    else:
        s["q"] = (torch.randn((total, hq, d), generator=gen, device=DEVICE) * c["gain"]).to(wide)
        s["out"] = torch.zeros((total, hq, d), dtype=wide, device=DEVICE)
    return s


def prepare(case, seed):
    s = _inputs(dict(case), seed)
    if own:
        _prepare_own(s)
    return s


# ---- the plain forms ------------------------------------------------------------------------------


def _dense(s, name, scale, values):
    """A cache's tokens, [sequences][heads][tokens][d] in 32 bits, gathered by the tables."""
    c = s["c"]
    x = s[name][s["tables"].clamp(min=0).long()]  # [sequences][blocks][heads][..]
    if c["dtype"] == "mx4":
        codes, e = _mx4_split(x, c["d"], values)
        lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEVICE)
        x = (lut[codes.int()].unflatten(-1, (-1, GROUP)) * _power(e)[..., None]).flatten(-2)
    else:
        x = x.view(torch.float8_e4m3fn).float() if c["dtype"] == "fp8" else x.float()
        if scale is not None:
            x = x * scale[s["tables"].clamp(min=0).long()][:, :, None, None, None]
        x = x.transpose(-1, -2) if values else x
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3).contiguous()


def _attention(s):
    """Softmax attention of the new tokens, in 32 bits over every sequence padded to the longest."""
    c = s["c"]
    n, hq, hkv, d, most = c["seqs"], c["hq"], c["hkv"], c["d"], s["max_new"]
    g = hq // hkv
    offs, lens = s["offs"].long(), s["lens"].long()
    new = offs[1:] - offs[:-1]
    i = torch.arange(most, device=DEVICE)
    at = (offs[:-1, None] + i).clamp(max=s["total"] - 1)
    q = s["q"][at].float().reshape(n, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * g, d)
    k = _dense(s, "k", s["ks"], False).transpose(-1, -2).contiguous()
    last = (lens - new)[:, None] + i  # the last token that query i sees
    hidden = torch.arange(k.shape[-1], device=DEVICE) > last[:, :, None]
    p = torch.matmul(q, k)
    del k
    p *= 1.0 / math.sqrt(d)
    p.view(n, hkv, most, g, -1).masked_fill_(hidden[:, None, :, None], -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    total = p.sum(-1, keepdim=True)
    v = _dense(s, "v", s["vs"], True)
    v.masked_fill_((torch.arange(v.shape[2], device=DEVICE) >= lens[:, None])[:, None, :, None], 0.0)  # unused slots
    out = (torch.matmul(p, v) / total).reshape(n, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(n, most, hq, d)
    return out[i < new[:, None]].to(s["out"].dtype)


def _rotate(x, cos, sin, c):
    half, rot = c["rot"] // 2, c["rot"]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, half), slice(half, rot))
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _store(s, name, scale, x, block, slot, values):
    """Tokens x [t][heads][d] in 32 bits into slots of blocks of a cache."""
    c, cache, d = s["c"], s[name], s["c"]["d"]
    if c["dtype"] == "mx4":
        codes, e = _mx4_split(cache[s["touched"]], d, values)
        codes, e = codes.contiguous(), e.contiguous()
        where = s["place"][block]
        codes[where, :, slot], e[where, :, slot] = _mx4(x)
        cache[s["touched"]] = _mx4_store(codes, e, values)
        return
    if c["dtype"] == "fp8":
        t = s["touched"]
        where, count = s["place"][block], len(t)
        top = torch.zeros(count, device=DEVICE).scatter_reduce_(0, where, x.abs().flatten(1).amax(1), "amax")
        first = torch.full((count,), BLOCK, device=DEVICE).scatter_reduce_(0, where, slot, "amin")
        old, fit = scale[t], top / FP8_MAX
        now = torch.where(first == 0, torch.where(top > 0, fit, torch.ones_like(fit)),
                          torch.where(top > FP8_MAX * old, fit, old))
        codes = cache[t].view(torch.float8_e4m3fn).float()
        again = (codes * old.view(-1, 1, 1, 1) / now.view(-1, 1, 1, 1)).clamp_(-FP8_MAX, FP8_MAX)
        early = torch.arange(BLOCK, device=DEVICE) < first[:, None]
        early = (early & (now != old)[:, None]).view((count, 1, 1, BLOCK) if values else (count, 1, BLOCK, 1))
        cache[t] = torch.where(early, again, codes).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[t] = now
        x = (x / now[where].view(-1, 1, 1)).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    if values:
        cache[block, :, :, slot] = x.to(cache.dtype)
    else:
        cache[block, :, slot] = x.to(cache.dtype)


def _append(s):
    c = s["c"]
    hq, hkv = c["hq"], c["hkv"]
    offs, lens = s["offs"].long(), s["lens"].long()
    t = torch.arange(s["total"], device=DEVICE)
    b = torch.searchsorted(offs, t, right=True) - 1
    pos = lens[b] - offs[b + 1] + t
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    x = s["qkv"].float()
    s["q_out"].copy_(_rotate(x[:, :hq], cos, sin, c))
    block, slot = s["tables"][b, pos // BLOCK].long(), pos % BLOCK
    s["place"] = torch.zeros(s["pool"], dtype=torch.long, device=DEVICE)
    s["place"][s["touched"]] = torch.arange(len(s["touched"]), device=DEVICE)
    _store(s, "k", s["ks"], _rotate(x[:, hq:hq + hkv], cos, sin, c), block, slot, False)
    _store(s, "v", s["vs"], x[:, hq + hkv:], block, slot, True)


def _held(s):
    """What an append leaves, as values: E4M3 codes by their own type, E2M1 codes (all of them E4M3 values too) through
    a table of two to a byte, and the scale bytes of the blocks written."""
    c = s["c"]
    if c["dtype"] == "fp8":
        return {"q": s["q_out"], "k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn),
                "ks": s["ks"], "vs": s["vs"]}
    if c["dtype"] != "mx4":
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    n = BLOCK * c["d"] // 2
    lut = _pairs()
    found = {"q": s["q_out"]}
    for name in ("k", "v"):
        x = s[name][s["touched"]]
        found[name] = lut[x[..., :n].int()].view(torch.float8_e4m3fn)
        found[name + "s"] = x[..., n:].contiguous().view(torch.float8_e8m0fnu)
    return found


_LUT = []


def _pairs():
    """The two E2M1 values of a byte as E4M3 codes, lower half first (a constant table)."""
    if not _LUT:
        v = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEVICE).to(torch.float8_e4m3fn).view(torch.uint8)
        byte = torch.arange(256, device=DEVICE)
        _LUT.append(torch.stack([v[byte & 15], v[byte >> 4]], -1).contiguous().view(torch.int16)[:, 0].contiguous())
    return _LUT[0]


def run(state):
    s, kind = state, state["c"]["kind"]
    if kind == "rope":
        if own:
            _own_append(s)
        else:
            _append(s)
        return _held(s)
    if own:
        _own_attention(s)
        return {"out": s["out"]}
    return {"out": _attention(s)}


# ---- the framework's calls --------------------------------------------------------------------------


def _prepare_own(s):
    """The handle of the shared prefixes, and the workspace."""
    from paper_2509_00195_amd import tts as T

    c = s["c"]
    wide = "f32" if c["dtype"] == "f32" else "bf16"
    s["desc"] = desc = T.make_desc(c["hq"], c["hkv"], c["d"], BLOCK, wide, c["dtype"], wide)
    size = 0
    if c["kind"] in ("prefix", "verify"):
        req = np.arange(0, c["seqs"] + 1, c["beams"], dtype=np.int32)
        s["meta"] = T.tts_build_verify_meta(req, s["tables_h"], s["lens_h"], c["q_hi"], BLOCK, s["pool"], desc=desc) \
            if c["kind"] == "verify" else T.tts_build_prefix_meta(req, s["tables_h"], s["lens_h"], BLOCK, s["pool"], desc=desc)
        size = T.tts_prefix_decode_workspace_size(desc, s["meta"])
    elif c["kind"] == "paged":
        size = T.tts_paged_decode_workspace_size(desc, c["seqs"], s["max_len"])
    elif c["kind"] == "prefill":
        size = T.tts_paged_prefill_workspace_size(desc, c["seqs"], s["total"], s["max_len"])
    s["ws"] = torch.empty(max(1, size), dtype=torch.uint8, device=DEVICE)


def _own_append(s):
    from paper_2509_00195_amd import tts as T

    c = s["c"]
    hq, hkv = c["hq"], c["hkv"]
    x = s["qkv"]
    rope = T.make_rope(s["cos"], s["sin"], interleaved=c["inter"])
    T.tts_rope_append_kv(s["desc"], c["seqs"], s["total"], x[:, hq:hq + hkv], x[:, hq + hkv:], s["tables"],
                         s["tables"].shape[1], s["lens"], s["pool"], s["k"], s["v"], s["ks"], s["vs"], rope=rope,
                         q=x[:, :hq], q_out=s["q_out"], tok_offsets=s["offs"] if c["q_hi"] > 1 else None)


def _own_attention(s):
    from paper_2509_00195_amd import tts as T

    c, desc, t = s["c"], s["desc"], s["tables"]
    cache = (s["k"], s["v"], s["ks"], s["vs"])
    if c["kind"] == "prefill":
        T.tts_paged_prefill_attn(desc, c["seqs"], s["total"], s["offs"], s["q"], *cache, t, t.shape[1], s["lens"],
                                 s["max_len"], s["pool"], s["out"], s["ws"], s["ws"].numel())
    elif c["kind"] == "paged":
        T.tts_paged_decode_attn(desc, c["seqs"], s["q"], *cache, t, t.shape[1], s["lens"], s["max_len"], s["pool"],
                                s["out"], s["ws"], s["ws"].numel())
    else:
        call = T.tts_prefix_verify_attn if c["kind"] == "verify" else T.tts_prefix_decode_attn
        call(desc, s["meta"], s["q"], *cache, t, t.shape[1], s["lens"], s["pool"], s["out"], s["ws"], s["ws"].numel())


# ---- what a pass cannot do without -------------------------------------------------------------------


def work(case):
    c = case
    eb = {"f32": 4.0, "bf16": 2.0, "fp8": 1.0, "mx4": 0.53125}[c["dtype"]]
    qb = 4 if c["dtype"] == "f32" else 2
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    new, lens = (x.astype(np.int64) for x in _lengths(c))
    total = int(new.sum())
    if c["kind"] == "rope":
        tables = min(total, int(lens.max())) * c["rot"] * 4
        return {"bytes": int(total * ((2 * hq + 2 * hkv) * d * qb + 2 * hkv * d * eb) + tables),
                "flops": 3 * total * (hq + hkv) * c["rot"]}
    tokens = int(lens.sum())
    if c["kind"] in ("prefix", "verify"):
        tokens = min(tokens, _tables(c, lens, 0)[2] * BLOCK)  # every block once
    seen = int((new * lens - new * (new - 1) // 2).sum())  # (query, visible token) pairs
    return {"bytes": int(tokens * 2 * hkv * d * eb + 2 * total * hq * d * qb), "flops": 4 * d * hq * seen}


# ---- 64 bits -------------------------------------------------------------------------------------------


def _nearest(x, values):
    """The nearest of increasing values of one sign, ties to the even place; x: magnitudes."""
    v = torch.tensor(values, dtype=torch.float64, device=DEVICE)
    hi = torch.searchsorted(v, x.contiguous()).clamp(1, len(values) - 1)
    lo = hi - 1
    down, up = x - v[lo], v[hi] - x
    pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return v[torch.where(x <= 0, torch.zeros_like(pick), pick)]


def _e4m3():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    return codes.double().tolist()


def _blocks64(s, name, scale, ids, values):
    """Blocks ids of a cache as [heads][tokens][d] values in 64 bits."""
    c = s["c"]
    x, d, hkv = s[name][ids], c["d"], c["hkv"]
    if c["dtype"] == "mx4":
        n = BLOCK * d // 2
        byte = x[..., :n].long()
        code = torch.empty((*byte.shape[:-1], 2 * n), dtype=torch.long, device=DEVICE)
        code[..., 0::2], code[..., 1::2] = byte % 16, byte // 16
        y = torch.tensor(E2M1, dtype=torch.float64, device=DEVICE)[code % 8] * (1 - 2 * (code // 8)).double()
        e = torch.exp2(x[..., n:].double() - 127.0)
        if values:
            y = y.view(-1, hkv, d // GROUP, GROUP, BLOCK) * e.view(-1, hkv, d // GROUP, 1, BLOCK)
            y = y.view(-1, hkv, d, BLOCK).transpose(2, 3)
        else:
            y = (y.view(-1, hkv, BLOCK, d // GROUP, GROUP) * e.view(-1, hkv, BLOCK, d // GROUP, 1)).view(-1, hkv, BLOCK, d)
    else:
        y = x.view(torch.float8_e4m3fn).float().double() if c["dtype"] == "fp8" else x.double()
        y = y * scale[ids].double().view(-1, 1, 1, 1) if scale is not None else y
        y = y.transpose(2, 3) if values else y
    return y.transpose(0, 1).reshape(hkv, -1, d)


def _exact_attention(s):
    c = s["c"]
    hq, hkv, d, g = c["hq"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    offs, tables = s["offs"].tolist(), s["tables"].long()
    out = torch.zeros((s["total"], hq, d), dtype=torch.float64, device=DEVICE)
    for b in range(c["seqs"]):
        ln, n = int(s["lens_h"][b]), offs[b + 1] - offs[b]
        ids = tables[b, : -(-ln // BLOCK)]
        k = _blocks64(s, "k", s["ks"], ids, False)[:, :ln].transpose(1, 2).contiguous()
        v = _blocks64(s, "v", s["vs"], ids, True)[:, :ln].contiguous()
        for a in range(0, n, 1024):
            m = min(1024, n - a)
            q = s["q"][offs[b] + a: offs[b] + a + m].double().view(m, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * m, d)
            score = torch.matmul(q.contiguous(), k).div_(math.sqrt(d)).view(hkv, g, m, ln)
            seen = torch.arange(ln, device=DEVICE) <= (ln - n + a + torch.arange(m, device=DEVICE))[:, None]
            p = torch.softmax(score.masked_fill_(~seen, -math.inf), -1)
            y = torch.matmul(p.view(hkv, g * m, ln), v).view(hkv, g, m, d)
            out[offs[b] + a: offs[b] + a + m] = y.permute(2, 0, 1, 3).reshape(m, hq, d)
    return {"out": out}


def _exact_append(s):
    c = s["c"]
    hq, hkv, d, rot, half = c["hq"], c["hkv"], c["d"], c["rot"], c["rot"] // 2
    offs = s["offs"].tolist()
    pos = torch.cat([torch.arange(int(ln) - (e - a), int(ln)) for a, e, ln in zip(offs, offs[1:], s["lens_h"])]).to(DEVICE)
    seq = torch.cat([torch.full((e - a,), i) for i, (a, e) in enumerate(zip(offs, offs[1:]))]).to(DEVICE)
    block, slot = s["tables"].long()[seq, pos // BLOCK], pos % BLOCK
    # A rotation is a product with exp(i angle) of the pair as a complex number.
    turn = torch.complex(s["cos"].double()[pos], s["sin"].double()[pos])[:, None]
    x = s["qkv"].double()
    y = x.clone()
    pair = x[:, : hq + hkv, :rot]
    z = (torch.complex(pair[..., 0::2], pair[..., 1::2]) if c["inter"] else torch.complex(pair[..., :half], pair[..., half:])) * turn
    y[:, : hq + hkv, :rot] = torch.stack([z.real, z.imag], -1 if c["inter"] else -2).reshape(pair.shape)
    found = {"q": y[:, :hq]}
    for name, new, values in (("k", y[:, hq:hq + hkv], False), ("v", y[:, hq + hkv:], True)):
        if c["dtype"] in ("f32", "bf16"):
            cache = s[name].double()
            if values:
                cache[block, :, :, slot] = new
            else:
                cache[block, :, slot] = new
            found[name] = cache
            continue
        if c["dtype"] == "fp8":
            scale = s[name + "s"].double()
            for a, e, ln in zip(offs, offs[1:], s["lens_h"]):
                start = int(ln) - (e - a)
                for at in range(start // BLOCK, -(-int(ln) // BLOCK)):
                    i0, i1 = max(a, a + at * BLOCK - start), min(e, a + (at + 1) * BLOCK - start)
                    top, p = float(new[i0:i1].abs().max()), int(block[i0])
                    if int(slot[i0]) == 0:
                        scale[p] = top / FP8_MAX if top > 0 else 1.0
                    else:
                        scale[p] = max(float(scale[p]), top / FP8_MAX)
            found[name + "s"], found[name] = scale, None
            continue
        codes, e = _mx4_split(s[name][s["touched"]], d, values)
        signed = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64, device=DEVICE)
        codes, e = signed[codes.long()].clone(), torch.exp2(e.double() - 127.0)
        where = torch.zeros(s["pool"], dtype=torch.long, device=DEVICE)
        where[s["touched"]] = torch.arange(len(s["touched"]), device=DEVICE)
        groups = new.reshape(len(pos), hkv, d // GROUP, GROUP)
        shared = torch.exp2(torch.floor(torch.log2(groups.abs().amax(-1))) - 2.0)
        m = groups / shared[..., None]
        codes[where[block], :, slot] = (_nearest(m.abs(), E2M1) * torch.sign(m)).reshape(len(pos), hkv, d)
        e[where[block], :, slot] = shared
        if values:
            codes, e = codes.transpose(-1, -2), e.transpose(-1, -2)
        found[name], found[name + "s"] = codes.flatten(-2), e.flatten(-2)
    return found


def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    return _exact_append(s) if c["kind"] == "rope" else _exact_attention(s)
