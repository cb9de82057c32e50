// KV-cache maintenance around the decode step: appending each beam's new
// token to its block (with the fp8 block-scale policy), appending chunks of
// tokens with their position rotation, and copying blocks for copy-on-write
// beam duplication.
//
// A decode step of the search writes one token per beam into the paged
// cache before attention reads it (the current token is part of seq_len),
// and a duplicated beam shares its parent's full blocks while its partially
// filled last block is copied (DuplicateThenTruncate, Sec. 3.1 and Alg. 1;
// the duplicates' speculative tokens are truncated, Sec. 4.1).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "tts_device.h"
#include "tts_kv.h"

namespace tts {
namespace {

constexpr int kKvThreads = 256;
constexpr int kSlots = 16;  // tokens per block

// Round-to-nearest-even OCP E4M3FN encoding of an fp32 value (already
// divided by its block scale), saturating at +-448 (code 0x7E); NaN gives
// 0x7F. Built from the format: subnormals are multiples of 2^-9 below 2^-6,
// normals keep 3 mantissa bits of the fp32 significand.
__device__ __forceinline__ uint32_t e4m3_encode(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const uint32_t sign = (u >> 24) & 0x80u;
  const float a = __builtin_fabsf(x);
  if (a != a) return 0x7Fu;
  if (a >= 448.f) return sign | 0x7Eu;
  if (a < 0.015625f) {  // 2^-6: subnormal codes q * 2^-9, q in [0, 8]
    const uint32_t q = static_cast<uint32_t>(__builtin_rintf(a * 512.f));  // exact scaling, RNE
    return sign | q;
  }
  const uint32_t ua = __builtin_bit_cast(uint32_t, a);
  int e = static_cast<int>(ua >> 23) - 127;  // -6 .. 8
  uint32_t keep = (ua >> 20) & 7u;
  const uint32_t rest = ua & 0xFFFFFu;
  if (rest > 0x80000u || (rest == 0x80000u && (keep & 1u))) ++keep;
  if (keep == 8u) {
    keep = 0;
    ++e;
  }
  return sign | (static_cast<uint32_t>(e + 7) << 3) | keep;
}

__device__ __forceinline__ float e4m3_decode(uint32_t code) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(code), 0);  // exact
}

__device__ __forceinline__ float block_max(float v, float* red) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  const int w = threadIdx.x >> 6;
  __syncthreads();  // red is free (a previous reduction is done with it)
  if ((threadIdx.x & 63) == 0) red[w] = v;
  __syncthreads();
  float m = red[0];
  for (int i = 1; i < kKvThreads / 64; ++i) m = fmaxf(m, red[i]);
  return m;
}

struct AppendParams {
  const void* k_new;  // [S][Hkv][D]: bf16 (fp32 caches: fp32)
  const void* v_new;
  const int32_t* block_tables;
  const int32_t* seq_lens;
  void* k_cache;  // [NB][Hkv][16][D]
  void* v_cache;  // [NB][Hkv][D][16]
  float* k_scale;
  float* v_scale;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t hkv;
  int32_t head_dim;
};

// Elements of a token that a thread holds in registers (tokens of more are
// read again from memory).
constexpr int kHeld = 4;

// Sixteen codes of a 16-byte word, each of the first n through the table
// (and code `at`, if it is one of them, replaced by `code`).
__device__ __forceinline__ uint4 map_codes(uint4 x, const uint8_t* lut, int n, int at, uint32_t code) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = 4 * i + k;
      const uint32_t c = (w[i] >> (8 * k)) & 0xFFu;
      r |= (j == at ? code : (j < n ? lut[c] : c)) << (8 * k);
    }
    w[i] = r;
  }
  return uint4{w[0], w[1], w[2], w[3]};
}

// One tensor (K or V) of one beam's new token into an fp8 block: element
// i = h * D + d of the token to slot `slot` of head h, dim d. The block's
// scale is set from the token when the token opens the block (slot 0); when
// a later token exceeds the range of the current scale the scale grows to
// fit it and the block's earlier codes are re-encoded under the new scale.
//
// Bound by its chain of round trips (length, table, scale, earlier codes;
// the token and its maximum travel beside them) and by the re-encoding: the
// 256 codes' new values are computed once, one per thread, into a table in
// LDS, and the earlier codes go through it sixteen at a time. 512 beams, 512
// values per token, sixteen tokens: 12.5 -> 6.7 us per call (a conversion, a
// product and a division per code, a byte at a time, and the token read
// after the table).
template <bool kV>
__device__ void append_fp8(const float (&held)[kHeld], float amax, const uint16_t* src, int n, int slot,
                           float* scale_p, uint8_t* blk, int D, uint8_t* lut) {
  // (A cache that starts at no multiple of 16 bytes is re-encoded by bytes.)
  const bool wide = (reinterpret_cast<uintptr_t>(blk) & 15) == 0;
  const float s_old = *scale_p;
  float s = s_old;
  bool requant = false;
  if (slot == 0) {
    s = amax > 0.f ? amax / 448.f : 1.f;
  } else if (amax > 448.f * s_old) {
    s = amax / 448.f;
    requant = true;
  }
  if (requant) {
    lut[threadIdx.x] = static_cast<uint8_t>(e4m3_encode(e4m3_decode(threadIdx.x) * s_old / s));
    __syncthreads();
    if constexpr (!kV) {
      // Rows of D codes: the earlier slots of a head are contiguous.
      const int per = slot * D / 16, total = n / D * per;
      for (int c = threadIdx.x; c < total; c += kKvThreads) {
        uint8_t* x = blk + (c / per) * kSlots * D + c % per * 16;
        if (wide)
          *reinterpret_cast<uint4*>(x) = map_codes(*reinterpret_cast<const uint4*>(x), lut, 16, -1, 0);
        else
          for (int j = 0; j < 16; ++j) x[j] = lut[x[j]];
      }
    }
  }
  for (int k = 0, i = threadIdx.x; i < n; ++k, i += kKvThreads) {
    float v = k < kHeld ? 0.f : bf16_to_f32(src[i]);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) v = k == j ? held[j] : v;
    const uint32_t code = e4m3_encode(v / s);
    if constexpr (kV) {
      // Row i holds the sixteen slots of one dimension.
      uint8_t* x = blk + static_cast<int64_t>(i) * kSlots;
      if (requant && wide) {
        *reinterpret_cast<uint4*>(x) = map_codes(*reinterpret_cast<const uint4*>(x), lut, slot, slot, code);
      } else {
        for (int j = 0; requant && j < slot; ++j) x[j] = lut[x[j]];
        x[slot] = static_cast<uint8_t>(code);
      }
    } else {
      blk[(static_cast<int64_t>(i / D) * kSlots + slot) * D + i % D] = static_cast<uint8_t>(code);
    }
  }
  __syncthreads();  // every thread has read s_old
  if (threadIdx.x == 0) *scale_p = s;
}

// Two workgroups per beam, one for K and one for V (their dependent steps
// run side by side): the beam's current token (position seq_len - 1) into
// slot (seq_len - 1) % 16 of its block. Beams with seq_len 0, a block index
// past the table row or a block id outside the pool write nothing.
template <int KV>  // 0 fp32, 1 bf16, 2 fp8
__global__ __launch_bounds__(kKvThreads) void append_kernel(AppendParams p) {
  __shared__ float red[kKvThreads / 64];
  __shared__ uint8_t lut[kKvThreads];
  typedef typename std::conditional<KV == 0, float, uint16_t>::type E;
  const int b = static_cast<int>(blockIdx.x >> 1);
  const bool is_v = (blockIdx.x & 1) != 0;
  const int D = p.head_dim, n = p.hkv * D;
  // The token is read beside the length and the table entry, not after them.
  const E* src = static_cast<const E*>(is_v ? p.v_new : p.k_new) + static_cast<int64_t>(b) * n;
  E tok[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = threadIdx.x + kKvThreads * k;
    tok[k] = i < n ? src[i] : E{};
  }
  const int L = p.seq_lens[b];
  if (L <= 0) return;
  const int t = L - 1;
  const int lb = t / kSlots, slot = t % kSlots;
  if (lb >= p.max_blocks) return;
  const int blk = p.block_tables[static_cast<int64_t>(b) * p.max_blocks + lb];
  float held[kHeld], a = 0.f;
  if constexpr (KV == 2) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      held[k] = bf16_to_f32(tok[k]);
      a = fmaxf(a, __builtin_fabsf(held[k]));
    }
    for (int i = threadIdx.x + kKvThreads * kHeld; i < n; i += kKvThreads)
      a = fmaxf(a, __builtin_fabsf(bf16_to_f32(src[i])));
    a = block_max(a, red);
  }
  if (blk < 0 || blk >= p.num_blocks) return;
  const int64_t base = static_cast<int64_t>(blk) * p.hkv;  // (block, head 0)
  if constexpr (KV == 2) {
    uint8_t* cache = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + base * kSlots * D;
    if (is_v)
      append_fp8<true>(held, a, src, n, slot, p.v_scale + blk, cache, D, lut);
    else
      append_fp8<false>(held, a, src, n, slot, p.k_scale + blk, cache, D, lut);
  } else {
    E* dst = static_cast<E*>(is_v ? p.v_cache : p.k_cache) + base * kSlots * D;
    for (int k = 0, i = threadIdx.x; i < n; ++k, i += kKvThreads) {
      E v = k < kHeld ? E{} : src[i];
#pragma unroll
      for (int j = 0; j < kHeld; ++j) v = k == j ? tok[j] : v;
      dst[is_v ? static_cast<int64_t>(i) * kSlots + slot
               : (static_cast<int64_t>(i / D) * kSlots + slot) * D + i % D] = v;
    }
  }
}

// ---- rotating append ---------------------------------------------------------
// A workgroup takes one part of one item, an item being one cache block of
// one sequence and the up to sixteen new tokens that go there, so that what
// a block shares (an fp8 scale, a byte of two 4-bit tokens, a line of a
// dim-major V row) has one writer and no atomics. Parts: the K rows of
// `heads_per` heads, the V rows of as many, kRopeTasks pieces of the query
// rows. Bound by memory for chunks (eight of 256 to 2,048 tokens, 28 over 4 heads of
// 128, 4-bit cache: 30.9 us, a copy of as many bytes 30.2), by the round
// trips (offsets, length, table and table rows, token) for a step's single
// tokens (16 sequences 4.9 us; 512 over an fp8 cache, whose earlier codes may
// have to be read and encoded again, 10.1 us).
//
// The products of the rotation and their sum are rounded one by one (no
// fused multiply-add), so codes do not depend on how the compiler contracts.
constexpr int kRopeThreads = kKvThreads;

struct RopeItem {
  int seq, n;     // sequence, tokens of it in this block
  int row;        // first token's row of q, k_new, v_new
  int pos, slot;  // its index in the sequence, its slot in the block
  int blk;        // physical block, -1: nothing is stored
  bool bad;       // the sequence is shorter than its new tokens: NaN queries
};

// The item's sequence: items [f(b), f(b + 1)) belong to sequence b, with
// f(b) = offsets[b] / 16 + 2 b. A sequence of n > 0 new tokens touches at
// most (n + 30) / 16 blocks (rounded down), which is at most
// f(b + 1) - f(b); the items past its last block are empty.
__device__ __forceinline__ RopeItem rope_item(const RopeParams& p, int64_t item) {
  RopeItem it{0, 0, 0, 0, 0, -1, false};
  int64_t j = 0;
  int t0, t1;
  if (p.tok_offsets) {
    auto first = [&](int64_t b) { return (static_cast<int64_t>(p.tok_offsets[b]) >> 4) + 2 * b; };
    it.seq = find_seq(p.num_seqs, item, first);
    t0 = p.tok_offsets[it.seq];
    t1 = p.tok_offsets[it.seq + 1];
    j = item - first(it.seq);
    if (t0 < 0 || t1 < t0 || t1 > p.num_tokens || j < 0) return it;
  } else {
    it.seq = static_cast<int>(item);
    t0 = it.seq;
    t1 = t0 + 1;
  }
  const int n = t1 - t0, len = p.seq_lens[it.seq];
  if (len <= 0 || n == 0) return it;  // idle
  it.bad = len < n;
  const int pos0 = it.bad ? 0 : len - n;
  const int64_t lb = pos0 / kSlots + j, last = static_cast<int64_t>(pos0) + n;
  if (lb * kSlots >= last) return it;
  it.pos = lb * kSlots > pos0 ? static_cast<int>(lb * kSlots) : pos0;
  it.slot = it.pos % kSlots;
  it.n = static_cast<int>((lb + 1) * kSlots < last ? (lb + 1) * kSlots : last) - it.pos;
  it.row = t0 + it.pos - pos0;
  if (!it.bad && lb < p.max_blocks) {
    it.blk = p.block_tables[static_cast<int64_t>(it.seq) * p.max_blocks + lb];
    if (it.blk < 0 || it.blk >= p.num_blocks) it.blk = -1;
  }
  return it;
}

// W consecutive elements of a token.
template <int W>
__device__ __forceinline__ void load_elems(const uint16_t* src, float (&x)[W]) {
  if constexpr (W == 8) {
    const uint4 t = *reinterpret_cast<const uint4*>(src);
    const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = bf16_to_f32(src[i]);
  }
}
template <int W>
__device__ __forceinline__ void load_elems(const float* src, float (&x)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    if constexpr (W >= 4) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(src + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[i + k] = t[k];
    } else {
      x[i] = src[i];
    }
  }
}
template <int W>
__device__ __forceinline__ void store_elems(uint16_t* dst, const float (&x)[W]) {
  if constexpr (W == 8)
    *reinterpret_cast<uint4*>(dst) = uint4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                           pack_bf16x2(x[6], x[7])};
  else
#pragma unroll
    for (int i = 0; i < W; ++i) dst[i] = static_cast<uint16_t>(pack_bf16x2(x[i], x[i]));
}
template <int W>
__device__ __forceinline__ void store_elems(float* dst, const float (&x)[W]) {
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    if constexpr (W >= 4)
      *reinterpret_cast<f32x4*>(dst + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
    else
      dst[i] = x[i];
  }
}

// One unit of a row of a head: W rotated pairs, or W elements passed through
// (interleaved and W > 1: W elements, which are W / 2 pairs or passed).
// Elements at[0] .. + W and, for two-part units, at[1] .. + W.
template <int W>
struct RopeUnit {
  int parts, at[2];
  float x[2][W];
};

template <int W>
__device__ __forceinline__ int rope_units(const RopeParams& p) {
  const int passed = (p.head_dim - p.rot) / W;
  return (p.interleaved && W > 1 ? p.rot / W : p.rot / 2 / W) + passed;
}

template <int W, typename E>
__device__ __forceinline__ RopeUnit<W> rope_unit(const RopeParams& p, const E* src, int u, const float* cos,
                                                 const float* sin) {
#pragma clang fp contract(off)
  RopeUnit<W> r;
  const int half = p.rot / 2, turned = p.interleaved && W > 1 ? p.rot / W : half / W;
  if (u >= turned) {
    r.parts = 1;
    r.at[0] = p.rot + (u - turned) * W;
    load_elems<W>(src + r.at[0], r.x[0]);
  } else if (W > 1 && p.interleaved) {
    constexpr int kPairs = W > 1 ? W / 2 : 1;
    r.parts = 1;
    r.at[0] = u * W;
    float x[W], c[kPairs], s[kPairs];
    load_elems<W>(src + u * W, x);
    load_elems<kPairs>(cos + u * kPairs, c);
    load_elems<kPairs>(sin + u * kPairs, s);
#pragma unroll
    for (int i = 0; i + 1 < W; i += 2) {
      const float xc = x[i] * c[i / 2], ys = x[i + 1] * s[i / 2], yc = x[i + 1] * c[i / 2], xs = x[i] * s[i / 2];
      r.x[0][i] = xc - ys;
      r.x[0][i + 1] = yc + xs;
    }
  } else {
    r.parts = 2;
    r.at[0] = p.interleaved ? 2 * u : u * W;
    r.at[1] = p.interleaved ? 2 * u + 1 : half + u * W;
    float x[W], y[W], c[W], s[W];
    load_elems<W>(src + r.at[0], x);
    load_elems<W>(src + r.at[1], y);
    load_elems<W>(cos + u * W, c);
    load_elems<W>(sin + u * W, s);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float xc = x[i] * c[i], ys = y[i] * s[i], yc = y[i] * c[i], xs = x[i] * s[i];
      r.x[0][i] = xc - ys;
      r.x[1][i] = yc + xs;
    }
  }
  return r;
}

__device__ __forceinline__ int64_t rope_pos(const RopeParams& p, const RopeItem& it, int i) {
  return p.positions ? p.positions[it.row + i] : it.pos + i;
}

// The item's tokens whose position has a row of the tables (bit i: token i).
__device__ __forceinline__ uint32_t rope_tokens(const RopeParams& p, const RopeItem& it) {
  const int lane = threadIdx.x & 63;
  bool good = lane < it.n;
  if (good && p.rot > 0) {
    const int64_t at = rope_pos(p, it, lane);
    good = at >= 0 && at < p.max_pos;
  }
  return static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(good));
}

// Calls f(token, head - h0, unit) for the units of heads h0 .. h1 of the
// item's good tokens, with the unit rotated.
template <int W, typename E, typename F>
__device__ __forceinline__ void rope_each(const RopeParams& p, const RopeItem& it, uint32_t good, const E* src,
                                          int64_t stride, int h0, int h1, int first, int last, F f) {
  const int units = rope_units<W>(p), heads = h1 - h0, total = it.n * heads * units;
  const int end = last < total ? last : total;
  for (int i = first + static_cast<int>(threadIdx.x); i < end; i += kRopeThreads) {
    const int u = i % units, h = i / units % heads, t = i / units / heads;
    if (!((good >> t) & 1u)) continue;
    const int64_t at = p.rot > 0 ? rope_pos(p, it, t) * (p.rot / 2) : 0;
    f(t, h, rope_unit<W>(p, src + (it.row + t) * stride + static_cast<int64_t>(h0 + h) * p.head_dim, u, p.cos + at,
                         p.sin + at));
  }
}

// Query rows: pieces [first, first + kRopeTasks) of the item's.
template <int W, typename E>
__device__ __forceinline__ void rope_query(const RopeParams& p, const RopeItem& it, uint32_t good, int part) {
  E* out = static_cast<E*>(p.q_out);
  const int first = part * kRopeTasks;
  if (it.bad || good != (1u << it.n) - 1u) {
    // NaN rows (all of a bad sequence's, else the tokens without a position), written by the first part.
    const float qnan[1] = {__builtin_nanf("")};
    const int row = p.hq * p.head_dim;
    for (int t = 0; part == 0 && t < it.n; ++t)
      if (it.bad || !((good >> t) & 1u))
        for (int i = threadIdx.x; i < row; i += kRopeThreads)
          store_elems<1>(out + static_cast<int64_t>(it.row + t) * row + i, qnan);
    if (it.bad) return;
  }
  rope_each<W>(p, it, good, static_cast<const E*>(p.q), p.q_stride, 0, p.hq, first, first + kRopeTasks,
               [&](int t, int h, const RopeUnit<W>& r) {
                 E* dst = out + (static_cast<int64_t>(it.row + t) * p.hq + h) * p.head_dim;
                 store_elems<W>(dst + r.at[0], r.x[0]);
                 if (r.parts == 2) store_elems<W>(dst + r.at[1], r.x[1]);
               });
}

// The scale of an fp8 block after the item's tokens, of largest magnitude
// `top`: set by them when they open the block, raised to fit them when they
// exceed it. `lut`: the earlier codes' new values, when it is raised.
__device__ __forceinline__ float fp8_scale(float top, float old, bool opens, bool* again, uint8_t* lut) {
  *again = !opens && top > 448.f * old;
  const float s = opens ? (top > 0.f ? top / 448.f : 1.f) : (*again ? top / 448.f : old);
  if (*again) lut[threadIdx.x] = static_cast<uint8_t>(e4m3_encode(e4m3_decode(threadIdx.x) * old / s));
  __syncthreads();
  return s;
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

// The scale byte of a group of largest magnitude `top` (bits): 2 to the
// power floor(log2 top) - 2, so that top / scale lies in [4, 8) (E2M1
// reaches 6; above 5 a value saturates or rounds to it). Infinities and
// NaN: 255, which makes the group's values NaN.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : (e > 3u ? e - 2u : 1u);
}

// E2M1 codes (nearest, ties to even, saturating) of eight values over the scale.
__device__ __forceinline__ uint32_t mx_encode(const float (&x)[8], uint32_t scale) {
  if (scale == 255u) return 0u;
  const float s = mx_scale<0>(scale);
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

// Scale byte and codes of eight of a group's 32 values, four adjacent lanes
// to a group (all four call together).
__device__ __forceinline__ uint32_t mx_quantise(const float (&x)[8], uint32_t* scale) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = top > abs_bits(x[i]) ? top : abs_bits(x[i]);
  for (int o = 1; o < 4; o <<= 1) {
    const uint32_t y = __shfl_xor(top, o);
    top = top > y ? top : y;
  }
  *scale = mx_scale_byte(top);
  return mx_encode(x, *scale);
}

// K rows of heads h0 .. h1.
template <int KV, int W, typename E>
__device__ __forceinline__ void rope_keys(const RopeParams& p, const RopeItem& it, uint32_t good, int h0, int h1,
                                          void* lds, float* red) {
  const int D = p.head_dim;
  const E* src = static_cast<const E*>(p.k_new);
  constexpr int kAll = 0x7FFFFFFF;
  if constexpr (KV == kKvF32 || KV == kKvBf16) {
    E* blk = static_cast<E*>(p.k_cache) + (static_cast<int64_t>(it.blk) * p.hkv + h0) * kSlots * D;
    rope_each<W>(p, it, good, src, p.k_stride, h0, h1, 0, kAll, [&](int t, int h, const RopeUnit<W>& r) {
      E* dst = blk + (h * kSlots + it.slot + t) * D;
      store_elems<W>(dst + r.at[0], r.x[0]);
      if (r.parts == 2) store_elems<W>(dst + r.at[1], r.x[1]);
    });
  } else if constexpr (KV == kKvFp8) {
    uint8_t* lut = static_cast<uint8_t*>(lds);
    const float old = p.k_scale[it.blk];
    float top = 0.f;
    rope_each<W>(p, it, good, src, p.k_stride, h0, h1, 0, kAll, [&](int, int, const RopeUnit<W>& r) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < W; ++i) top = k < r.parts ? fmaxf(top, __builtin_fabsf(r.x[k][i])) : top;
    });
    top = block_max(top, red);
    bool again;
    const float s = fp8_scale(top, old, it.slot == 0, &again, lut);
    uint8_t* blk = static_cast<uint8_t*>(p.k_cache) + static_cast<int64_t>(it.blk) * p.hkv * kSlots * D;
    if (again) {
      const int per = it.slot * D / 16, total = p.hkv * per;
      for (int c = threadIdx.x; c < total; c += kRopeThreads) {
        uint4* x = reinterpret_cast<uint4*>(blk + c / per * kSlots * D) + c % per;
        *x = map_codes(*x, lut, 16, -1, 0);
      }
    }
    rope_each<W>(p, it, good, src, p.k_stride, h0, h1, 0, kAll, [&](int t, int h, const RopeUnit<W>& r) {
      uint8_t* dst = blk + (h * kSlots + it.slot + t) * D;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (k >= r.parts) continue;
        uint32_t c[W];
#pragma unroll
        for (int i = 0; i < W; ++i) c[i] = e4m3_encode(r.x[k][i] / s);
        if constexpr (W == 8)
          *reinterpret_cast<uint2*>(dst + r.at[k]) = uint2{c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24,
                                                           c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24};
        else
          for (int i = 0; i < W; ++i) dst[r.at[k] + i] = static_cast<uint8_t>(c[i]);
      }
    });
    if (threadIdx.x == 0) p.k_scale[it.blk] = s;  // (read by every thread before block_max's barriers)
  } else {
    // Rotated rows in LDS, then four lanes to a group of 32 dims.
    float* tile = static_cast<float*>(lds);
    const int heads = h1 - h0;
    rope_each<W>(p, it, good, src, p.k_stride, h0, h1, 0, kAll, [&](int t, int h, const RopeUnit<W>& r) {
      float* dst = tile + (t * heads + h) * D;
      store_elems<W>(dst + r.at[0], r.x[0]);
      if (r.parts == 2) store_elems<W>(dst + r.at[1], r.x[1]);
    });
    __syncthreads();
    const int code_bytes = kSlots * D / 2, blk_bytes = code_bytes + kSlots * D / kMxGroup;
    uint8_t* blk = static_cast<uint8_t*>(p.k_cache) + (static_cast<int64_t>(it.blk) * p.hkv + h0) * blk_bytes;
    const int pieces = D / 8, total = it.n * heads * pieces;  // (a multiple of 8: groups are whole)
    for (int i = threadIdx.x; i < total; i += kRopeThreads) {
      const int piece = i % pieces, h = i / pieces % heads, t = i / pieces / heads;
      float x[8];
      load_elems<8>(tile + i * 8, x);
      uint32_t scale;
      const uint32_t codes = mx_quantise(x, &scale);
      if (!((good >> t) & 1u)) continue;
      uint8_t* b = blk + static_cast<int64_t>(h) * blk_bytes;
      *reinterpret_cast<uint32_t*>(b + ((it.slot + t) * D + 8 * piece) / 2) = codes;
      if (i % 4 == 0) b[code_bytes + ((it.slot + t) * D + 8 * piece) / kMxGroup] = static_cast<uint8_t>(scale);
    }
  }
}

// V rows of heads h0 .. h1: a dim's tokens lie side by side in the cache, so
// a thread takes dims (kVw of them) with all of the item's tokens.
template <int KV, int kVw, typename E>
__device__ __forceinline__ void rope_values(const RopeParams& p, const RopeItem& it, uint32_t good, int h0, int h1,
                                            void* lds, float* red) {
  const int D = p.head_dim, heads = h1 - h0;
  const E* src = static_cast<const E*>(p.v_new) + it.row * p.v_stride + static_cast<int64_t>(h0) * D;
  typedef E Vec __attribute__((ext_vector_type(kVw)));
  const bool full = good == 0xFFFFu;
  const uint32_t slots = good << it.slot;  // the block's slots that are written
  auto load = [&](int d, Vec (&x)[kSlots]) {  // by slot
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      Vec v = Vec(0);
      if ((slots >> k) & 1u) v = *reinterpret_cast<const Vec*>(src + (k - it.slot) * p.v_stride + d);
      x[k] = v;
    }
  };
  if constexpr (KV == kKvF32 || KV == kKvBf16) {
    E* blk = static_cast<E*>(p.v_cache) + (static_cast<int64_t>(it.blk) * p.hkv + h0) * kSlots * D;
    for (int d = threadIdx.x * kVw; d < heads * D; d += kRopeThreads * kVw) {
      Vec x[kSlots];
      load(d, x);
#pragma unroll
      for (int e = 0; e < kVw; ++e) {
        E* dst = blk + static_cast<int64_t>(d + e) * kSlots;
        if (full) {
          constexpr int kPer = 16 / sizeof(E);
          typedef E Out __attribute__((ext_vector_type(kPer)));
#pragma unroll
          for (int k = 0; k < kSlots; k += kPer) {
            Out o;
#pragma unroll
            for (int i = 0; i < kPer; ++i) o[i] = x[k + i][e];
            *reinterpret_cast<Out*>(dst + k) = o;
          }
        } else {
#pragma unroll
          for (int k = 0; k < kSlots; ++k)
            if ((slots >> k) & 1u) dst[k] = x[k][e];
        }
      }
    }
  } else if constexpr (KV == kKvFp8) {
    uint8_t* lut = static_cast<uint8_t*>(lds);
    const float old = p.v_scale[it.blk];
    float top = 0.f;
    for (int d = threadIdx.x * kVw; d < heads * D; d += kRopeThreads * kVw) {
      Vec x[kSlots];
      load(d, x);
#pragma unroll
      for (int k = 0; k < kSlots; ++k)
#pragma unroll
        for (int e = 0; e < kVw; ++e) top = fmaxf(top, __builtin_fabsf(bf16_to_f32(x[k][e])));
    }
    top = block_max(top, red);
    bool again;
    const float s = fp8_scale(top, old, it.slot == 0, &again, lut);
    uint8_t* blk = static_cast<uint8_t*>(p.v_cache) + (static_cast<int64_t>(it.blk) * p.hkv + h0) * kSlots * D;
    for (int d = threadIdx.x * kVw; d < heads * D; d += kRopeThreads * kVw) {
      Vec x[kSlots];
      load(d, x);
#pragma unroll
      for (int e = 0; e < kVw; ++e) {
        uint8_t* dst = blk + static_cast<int64_t>(d + e) * kSlots;
        if (!full && !again) {
#pragma unroll
          for (int k = 0; k < kSlots; ++k)
            if ((slots >> k) & 1u) dst[k] = static_cast<uint8_t>(e4m3_encode(bf16_to_f32(x[k][e]) / s));
          continue;
        }
        uint4 w = {0u, 0u, 0u, 0u};
        if (!full) w = map_codes(*reinterpret_cast<const uint4*>(dst), lut, it.slot, -1, 0);
        uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < kSlots; ++k)
          if ((slots >> k) & 1u)
            c[k / 4] = (c[k / 4] & ~(0xFFu << (8 * (k % 4)))) | e4m3_encode(bf16_to_f32(x[k][e]) / s) << (8 * (k % 4));
        *reinterpret_cast<uint4*>(dst) = uint4{c[0], c[1], c[2], c[3]};
      }
    }
    if (threadIdx.x == 0) p.v_scale[it.blk] = s;
  } else {
    // Codes in LDS, a byte each by (slot, dim); then eight bytes of a dim.
    uint8_t* tile = static_cast<uint8_t*>(lds);
    const int row = heads * D, code_bytes = kSlots * D / 2, blk_bytes = code_bytes + kSlots * D / kMxGroup;
    uint8_t* blk = static_cast<uint8_t*>(p.v_cache) + (static_cast<int64_t>(it.blk) * p.hkv + h0) * blk_bytes;
    const int pieces = row / 8;
    for (int i = threadIdx.x; i < it.n * pieces; i += kRopeThreads) {
      const int t = i / pieces, d = i % pieces * 8;
      float x[8];
      if constexpr (kVw == 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = bf16_to_f32(src[t * p.v_stride + d + k]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(src + t * p.v_stride + d + k);
          x[k] = __builtin_bit_cast(float, w << 16);
          x[k + 1] = __builtin_bit_cast(float, w & 0xFFFF0000u);
        }
      }
      uint32_t scale;
      const uint32_t codes = mx_quantise(x, &scale);
      uint2 bytes = {0u, 0u};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        bytes.x |= ((codes >> (4 * k)) & 15u) << (8 * k);
        bytes.y |= ((codes >> (4 * k + 16)) & 15u) << (8 * k);
      }
      *reinterpret_cast<uint2*>(tile + t * row + d) = bytes;
      if (i % 4 == 0 && ((good >> t) & 1u))
        blk[d / D * blk_bytes + code_bytes + d % D / kMxGroup * kSlots + it.slot + t] = static_cast<uint8_t>(scale);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < row; d += kRopeThreads) {
      uint2* dst = reinterpret_cast<uint2*>(blk + d / D * blk_bytes + d % D * (kSlots / 2));
      uint64_t w = 0u;
      if (!full) {
        const uint2 o = *dst;
        w = o.x | static_cast<uint64_t>(o.y) << 32;
      }
#pragma unroll
      for (int k = 0; k < kSlots; ++k)
        if ((slots >> k) & 1u)
          w = (w & ~(15ull << (4 * k))) | static_cast<uint64_t>(tile[(k - it.slot) * row + d]) << (4 * k);
      *dst = uint2{static_cast<uint32_t>(w), static_cast<uint32_t>(w >> 32)};
    }
  }
}

template <int KV>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(RopeParams p) {
  typedef typename std::conditional<KV == kKvF32, float, uint16_t>::type E;
  // 4-bit K: rotated rows in fp32; 4-bit V: codes; fp8: the codes' table.
  __shared__ __attribute__((aligned(16))) float lds[KV == kKvMx4 ? kRopeTile : (KV == kKvFp8 ? 64 : 4)];
  __shared__ float red[kRopeThreads / 64];
  const RopeItem it = rope_item(p, p.item0 + blockIdx.x);
  if (it.n == 0) return;
  const int part = static_cast<int>(blockIdx.y);
  const uint32_t good = rope_tokens(p, it);
  if (part >= 2 * p.kv_parts) {
    if (p.q_wide)
      rope_query<8, E>(p, it, good, part - 2 * p.kv_parts);
    else
      rope_query<1, E>(p, it, good, part - 2 * p.kv_parts);
    return;
  }
  if (it.blk < 0 || good == 0) return;
  const int h0 = part / 2 * p.heads_per, h1 = h0 + p.heads_per < p.hkv ? h0 + p.heads_per : p.hkv;
  if (part % 2 == 0) {
    if (p.k_wide)
      rope_keys<KV, 8, E>(p, it, good, h0, h1, lds, red);
    else
      rope_keys<KV, 1, E>(p, it, good, h0, h1, lds, red);
  } else {
    if (p.v_wide)
      rope_values<KV, 2, E>(p, it, good, h0, h1, lds, red);
    else
      rope_values<KV, 1, E>(p, it, good, h0, h1, lds, red);
  }
}

struct CopyParams {
  const int32_t* pairs;  // [n][2]: source, destination block
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  int64_t blk_bytes;  // bytes of one block of K (all KV heads), = V's
  int32_t num_blocks;
};

// K and V of every KV head (and the fp8 scales) of each pair's source block
// into its destination block. A workgroup copies one piece of kCopyBytes of
// one tensor, its two 16-byte loads per thread in flight together: bound by
// the memory and by the round trip to the pair and back (235 pairs of 32 KB:
// 8.1 -> 5.7 us; one workgroup per pair took four dependent rounds per
// tensor). Pairs naming a block outside the pool, or a block onto itself,
// copy nothing.
constexpr int kCopyBytes = kKvThreads * 32;
constexpr int kMaxGridY = 65535;

__global__ __launch_bounds__(kKvThreads) void copy_kernel(CopyParams p) {
  const int pair = static_cast<int>(blockIdx.y);
  const int src = p.pairs[2 * pair], dst = p.pairs[2 * pair + 1];
  if (src < 0 || src >= p.num_blocks || dst < 0 || dst >= p.num_blocks || src == dst) return;
  const bool is_v = (blockIdx.x & 1) != 0;
  unsigned char* cache = static_cast<unsigned char*>(is_v ? p.v_cache : p.k_cache);
  const int64_t n16 = p.blk_bytes / 16;
  const int64_t i0 = static_cast<int64_t>(blockIdx.x >> 1) * (kCopyBytes / 16) + threadIdx.x, i1 = i0 + kKvThreads;
  const uint4* s = reinterpret_cast<const uint4*>(cache + src * p.blk_bytes);
  uint4* d = reinterpret_cast<uint4*>(cache + dst * p.blk_bytes);
  uint4 x0, x1;
  if (i0 < n16) x0 = s[i0];
  if (i1 < n16) x1 = s[i1];
  if (i0 < n16) d[i0] = x0;
  if (i1 < n16) d[i1] = x1;
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.k_scale) {
    p.k_scale[dst] = p.k_scale[src];
    p.v_scale[dst] = p.v_scale[src];
  }
}

}  // namespace

// (A launch holds fewer than 2^32 threads: calls of more beams are made in
// runs.)
constexpr int kMaxAppendBeams = 0xFFFFFFFFu / kKvThreads / 2;

template <int KV>
static hipError_t launch_append_t(AppendParams p, int num_seqs, hipStream_t stream) {
  const int64_t token = static_cast<int64_t>(p.hkv) * p.head_dim * (KV == 0 ? 4 : 2);
  for (int left = num_seqs; left > 0; left -= kMaxAppendBeams) {
    const int n = left < kMaxAppendBeams ? left : kMaxAppendBeams;
    hipLaunchKernelGGL(append_kernel<KV>, dim3(2 * n), dim3(kKvThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.k_new = static_cast<const char*>(p.k_new) + n * token;
    p.v_new = static_cast<const char*>(p.v_new) + n * token;
    p.block_tables += static_cast<int64_t>(n) * p.max_blocks;
    p.seq_lens += n;
  }
  return hipSuccess;
}

hipError_t launch_append(const void* k_new, const void* v_new, const int32_t* block_tables, const int32_t* seq_lens,
                         void* k_cache, void* v_cache, float* k_scale, float* v_scale, int num_seqs, int max_blocks,
                         int num_blocks, int hkv, int head_dim, int kv_kind, hipStream_t stream) {
  const AppendParams p{k_new, v_new, block_tables, seq_lens, k_cache, v_cache, k_scale, v_scale,
                       max_blocks, num_blocks, hkv, head_dim};
  if (kv_kind == 0) return launch_append_t<0>(p, num_seqs, stream);
  if (kv_kind == 1) return launch_append_t<1>(p, num_seqs, stream);
  return launch_append_t<2>(p, num_seqs, stream);
}

// Whether rows at `ptr` of `stride` elements start at multiples of `bytes`.
static bool rows_at(const void* ptr, int64_t stride, int elem, int bytes) {
  return reinterpret_cast<uintptr_t>(ptr) % bytes == 0 && stride * elem % bytes == 0;
}

hipError_t launch_rope_append(RopeParams p, int kv_kind, hipStream_t stream) {
  const int elem = kv_kind == kKvF32 ? 4 : 2, half = p.rot / 2;
  // Eight elements at a time where rows, tables and the rotated part allow it.
  const bool parts8 = p.interleaved ? p.rot % 8 == 0 : half % 8 == 0;
  const bool tables8 = p.rot == 0 || (rows_at(p.cos, half, 4, 16) && rows_at(p.sin, half, 4, 16));
  p.q_wide = p.q && parts8 && tables8 && rows_at(p.q, p.q_stride, elem, 16) && rows_at(p.q_out, 0, elem, 16);
  p.k_wide = parts8 && tables8 && rows_at(p.k_new, p.k_stride, elem, 16);
  p.v_wide = rows_at(p.v_new, p.v_stride, elem, 2 * elem);
  const int most_tokens = p.tok_offsets ? kSlots : 1;
  // fp8: one scale for all heads of a block, so one part.
  p.heads_per = kRopeTile / (most_tokens * p.head_dim);
  if (kv_kind == kKvFp8 || p.heads_per > p.hkv) p.heads_per = p.hkv;
  p.kv_parts = (p.hkv + p.heads_per - 1) / p.heads_per;
  const int width = p.q_wide ? 8 : 1;
  const int64_t units = (p.interleaved && p.q_wide ? p.rot / width : half / width) + (p.head_dim - p.rot) / width;
  const int64_t q_parts = p.q ? (most_tokens * p.hq * units + kRopeTasks - 1) / kRopeTasks : 0;
  const int64_t parts = 2 * static_cast<int64_t>(p.kv_parts) + q_parts;
  if (parts > kMaxGridY) return hipErrorInvalidValue;
  const int64_t items = p.tok_offsets ? static_cast<int64_t>(p.num_tokens) / kSlots + 2 * static_cast<int64_t>(p.num_seqs)
                                      : p.num_seqs;
  const int64_t most = 0xFFFFFFFFll / kRopeThreads / parts;  // (a launch holds fewer than 2^32 threads)
  for (int64_t done = 0; done < items; done += most) {
    const int64_t n = items - done < most ? items - done : most;
    p.item0 = done;
    const dim3 grid(static_cast<unsigned>(n), static_cast<unsigned>(parts));
    switch (kv_kind) {
      case kKvF32: hipLaunchKernelGGL(rope_append_kernel<kKvF32>, grid, dim3(kRopeThreads), 0, stream, p); break;
      case kKvBf16: hipLaunchKernelGGL(rope_append_kernel<kKvBf16>, grid, dim3(kRopeThreads), 0, stream, p); break;
      case kKvFp8: hipLaunchKernelGGL(rope_append_kernel<kKvFp8>, grid, dim3(kRopeThreads), 0, stream, p); break;
      default: hipLaunchKernelGGL(rope_append_kernel<kKvMx4>, grid, dim3(kRopeThreads), 0, stream, p); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_copy_blocks(const int32_t* pairs, int num_pairs, void* k_cache, void* v_cache, float* k_scale,
                              float* v_scale, int64_t blk_bytes, int num_blocks, hipStream_t stream) {
  if (num_pairs <= 0) return hipSuccess;
  CopyParams p{pairs, k_cache, v_cache, k_scale, v_scale, blk_bytes, num_blocks};
  const int pieces = static_cast<int>((blk_bytes + kCopyBytes - 1) / kCopyBytes);
  // Pairs along the grid's second dimension, at most 65,535 to a launch.
  for (int done = 0; done < num_pairs; done += kMaxGridY) {
    const int n = num_pairs - done < kMaxGridY ? num_pairs - done : kMaxGridY;
    p.pairs = pairs + 2 * static_cast<int64_t>(done);
    hipLaunchKernelGGL(copy_kernel, dim3(2 * pieces, n), dim3(kKvThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace tts
