// HIP kernels (gfx950) of the ragged prefill attention: causal attention of
// each sequence's last tokens over its paged KV cache.
//
// A workgroup of four waves takes 128 query rows (tokens x query heads of one
// KV head) and walks the tokens that they see, a tile at a time: 64 tokens
// (fp32: 32) of K and V go from the paged cache through registers, converted
// to bf16 for fp8 and 4-bit caches, into one of two LDS buffers, while the
// waves work on the other; one barrier per tile. Each wave holds 32 rows:
//   S^T = K Q^T   : v_mfma_f32_32x32x16_bf16 (M = 32 tokens, N = 32 rows)
//   O^T += V^T P^T: the same (M = 32 dims, N = 32 rows, K = 16 tokens)
// K's rows are read in the order token_of, so that a lane's scores are those
// of 8 consecutive tokens per step of the second product: its B operand
// without an exchange between lanes. Values are dim-major in the cache, so
// the matching A operand is one 16-byte read.
//
// Softmax in one pass: exponentials against a reference per row that only
// moves (with a rescaling of the sums) when a tile's maximum exceeds it by
// more than kRefSlack: sums stay below 2^kRefSlack times the token count, far
// inside fp32's range, and the usual tile rescales nothing.
//
// LDS: a tile's 16-byte pieces lie fragment by fragment (one fragment is what
// the 64 lanes of a wave read for one operand), and inside a fragment at a
// place XORed with the piece's column, so that neither the stores (rows of
// the cache, 16 bytes per thread) nor the reads meet in a bank.
//
// Rounding: probabilities go to bf16 for the second product; the row's sum is
// that of the rounded ones (fp8 caches, whose probabilities are multiplied by
// V scales first: of the unrounded ones; dividing the rounded sum by the scale
// again, or folding the scale into the exponent, took 2 to 5% longer).
//
// Bound by the issue of matrix and vector instructions, which overlap only in
// part between the two waves of a SIMD: one sequence of 16,384 tokens, 28 over
// 4 heads of 128, takes 1.98 ms (972 TFLOP/s, 0.71 of a large bf16 matrix
// product here; cards differ by 5%); eight ragged prompts of 200 to 2048 111
// us; chunks over 8,000 to 16,000 tokens of an fp8 cache 166 us. Tried: eight waves in two groups
// that take turns at the matrix cores (4% faster at 16,384 tokens, fp8 chunks
// 264 us, D 64 98 instead of 78); the exponentials of one half of a tile
// between the products of the other (2.10 ms); four or eight LDS reads ahead
// instead of six (the same).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "tts_device.h"
#include "tts_prefill.h"

namespace tts {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kPfWaves = kPrefillRows / 32;
constexpr int kPfThreads = 64 * kPfWaves;
constexpr float kNegInf = -__builtin_inff();
constexpr float kRefSlack = 16.f;  // log2 units

template <int D, int KV>
struct PfGeo {
  // A piece as it comes from the cache.
  typedef typename std::conditional<
      KV == kKvMx4, uint32_t, typename std::conditional<KV == kKvFp8, uint2, uint4>::type>::type Raw;
  static constexpr bool f32 = KV == kKvF32;
  static constexpr int eb = f32 ? 4 : 2;                 // bytes of a staged element
  static constexpr int tokens = f32 ? 32 : 64;           // of a tile
  static constexpr int blocks = tokens / kTok;
  static constexpr int per = 16 / eb;                    // elements of a piece
  static constexpr int kcols = D / per;                  // pieces of a K row
  static constexpr int vcols = kTok / per;               // pieces of a V row
  static constexpr int blk_pieces = kTok * kcols;        // of K, and of V, in a block
  static constexpr int pieces = blocks * blk_pieces / kPfThreads;  // per thread and tensor
  static constexpr int tensor_bytes = tokens * D * eb;
  static constexpr int ksteps = kcols / 2;               // fragments of 32 tokens of K
  static constexpr int vsteps = tokens / (2 * per);      // fragments of 32 dims of V
};

// Token (of 32) in row m of the score product: see the header. (fp32 products
// take two tokens at a time, one per lane half: rows in their order.)
template <bool F32>
__device__ __forceinline__ int row_of_token(int t) {
  // token 16 a + 8 h + 4 b + j -> row 16 a + 8 b + 4 h + j
  return F32 ? t : (t & 0x13) | (t & 8) >> 1 | (t & 4) << 1;
}
// The token of accumulator register r in lane half 0 (half 1: 8, or 4, more).
template <bool F32>
__host__ __device__ constexpr int reg_token(int r) {
  return F32 ? 8 * (r >> 2) + (r & 3) : 16 * (r >> 3) + (r & 7);
}

// Byte of the LDS place of K piece (token of the tile, column) and V piece
// (dim, column of the tile's tokens).
template <typename G>
__device__ __forceinline__ int k_place(int tok, int col) {
  const int m = row_of_token<G::f32>(tok & 31);
  return ((tok >> 5) * G::ksteps + (col >> 1)) * 1024 + (col & 1) * 512 + ((m ^ (col & 15)) << 4);
}
template <typename G>
__device__ __forceinline__ int v_place(int dim, int col) {
  return ((dim >> 5) * G::vsteps + (col >> 1)) * 1024 + (col & 1) * 512 +
         (((dim & 31) ^ ((col & (G::vcols - 1)) * (16 / G::vcols))) << 4);
}

template <int KV, typename T>
__device__ __forceinline__ uint4 staged(T raw) {
  if constexpr (KV == kKvFp8)
    return fp8x8_to_bf16x8(raw);
  else
    return raw;
}

// Zeroes the elements from `keep` on.
template <bool F32>
__device__ __forceinline__ void keep_first(uint4& x, int keep) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32)
      w[i] = i < keep ? w[i] : 0u;
    else
      w[i] &= (2 * i < keep ? 0xFFFFu : 0u) | (2 * i + 1 < keep ? 0xFFFF0000u : 0u);
  }
}
// What an element that is not finite adds to the rows that see it.
enum : int { kBadNan = 0, kBadPos = 1, kBadNeg = 2, kBadKinds = 3 };

// Whether an element is not finite: its exponent is all ones. (Two bf16
// exponents at once: 0x8000 less what an exponent lacks keeps bit 15 only
// where nothing is lacking.)
template <bool F32>
__device__ __forceinline__ bool any_nonfinite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t all = 0u;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32)
      any = any || (w[i] & 0x7F800000u) == 0x7F800000u;
    else
      all |= 0x80008000u - (~w[i] & 0x7F807F80u);
  }
  return F32 ? any : (all & 0x80008000u) != 0u;
}

// Zeroes elements that are not finite, after f(place, kind) for each.
template <bool F32, typename F>
__device__ __forceinline__ void drop_nonfinite(uint4& x, F f) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&x);
  auto each = [&](uint32_t bits, int at) {  // bits: as fp32
    if ((bits & 0x7F800000u) != 0x7F800000u) return false;
    f(at, bits & 0x007FFFFFu ? kBadNan : (bits >> 31 ? kBadNeg : kBadPos));
    return true;
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      if (each(w[i], i)) w[i] = 0u;
    } else {
      if (each(w[i] << 16, 2 * i)) w[i] &= 0xFFFF0000u;
      if (each(w[i] & 0xFFFF0000u, 2 * i + 1)) w[i] &= 0xFFFFu;
    }
  }
}

// The larger of a lane's value and that of the same lane of the other half.
__device__ __forceinline__ float halves_max(float x) {
  // (In assembly: of the exchange builtin's two results this compiler keeps
  // one. The wait states are those it puts before the instruction.)
  float a = x, b = x;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}

struct PfItem {
  int seq, n, len;  // its new tokens and its length
  int row0;         // first row (token x g + head of the group) of the tile
  int64_t tok0;     // first new token's row of q
};

__device__ __forceinline__ PfItem prefill_item(const PrefillParams& p, int64_t item) {
  auto first = [&](int64_t b) { return static_cast<int64_t>(p.tok_offsets[b]) * p.g / kPrefillRows + b; };
  PfItem it;
  it.seq = find_seq(p.num_seqs, item, first);
  const int t0 = p.tok_offsets[it.seq], t1 = p.tok_offsets[it.seq + 1];
  it.tok0 = t0;
  it.n = t1 - t0;
  it.len = p.seq_lens[it.seq];
  const int64_t row0 = (item - first(it.seq)) * kPrefillRows;
  if (t0 < 0 || t1 < t0 || t1 > p.num_tokens || row0 < 0 || row0 >= static_cast<int64_t>(it.n) * p.g) it.n = 0;
  it.row0 = static_cast<int>(row0);
  return it;
}

// Schedule of kFrags fragments, each one LDS read and kProducts products: the
// reads go kAhead ahead (left to itself the compiler issues one or two, and
// every product waits for its operand): 16,384-token prompt 2237 -> 1980 us.
template <int kFrags, int kProducts>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kAhead = 6, kMfma = 0x008, kRead = 0x100;
  __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
  for (int i = 0; i < kFrags - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, kProducts, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, kProducts * kAhead, 0);
}

template <int D, int KV>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_kernel(PrefillParams p) {
  using G = PfGeo<D, KV>;
  using C = KvGeo<D, KV>;
  // K and V buffers of even and odd tiles.
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * G::tensor_bytes];
  // First token whose value in this dim is NaN, +inf, -inf (tiles with hidden tokens).
  __shared__ int bad_dim[kBadKinds][D];
  __shared__ int any_bad;  // whether there is one
  __shared__ int bad_tok;     // first token of a block that is not in the pool

  // Units in the order (tile of rows, split, KV head), the last tiles of a
  // call (which see the most tokens) first: KV heads side by side, so that
  // the XCDs (workgroups are dealt to them in turn) read few heads each.
  const int64_t unit = p.units - 1 - (p.unit0 + blockIdx.x);
  const int kvh = static_cast<int>(unit % p.hkv), split = static_cast<int>(unit / p.hkv % p.nsplit);
  const PfItem it = prefill_item(p, unit / p.hkv / p.nsplit);
  if (it.n <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nrows = it.n * p.g - it.row0 < kPrefillRows ? it.n * p.g - it.row0 : kPrefillRows;
  const int row = it.row0 + 32 * wave + ln;  // this lane's row of the sequence
  const bool active = 32 * wave + ln < nrows;
  const int64_t orow = (it.tok0 + row / p.g) * p.hq + kvh * p.g + row % p.g;
  // Tokens it sees: 0 .. lim. A sequence of length 0, one shorter than its
  // new tokens or longer than its table: no tokens.
  const bool bad = it.len > 0 && (it.len < it.n || it.len > p.max_seq_len || (it.len + kTok - 1) / kTok > p.max_blocks);
  const int before = it.len > 0 && !bad ? it.len - it.n : -1;  // tokens cached before the new ones
  const int lim = active && before >= 0 ? before + row / p.g : -1;
  const int wave_row = it.row0 + 32 * wave;
  const int first_lim = before >= 0 ? before + wave_row / p.g : -1;  // what the wave's first row sees,
  const int last_row = wave_row + 31 < it.row0 + nrows - 1 ? wave_row + 31 : it.row0 + nrows - 1;
  const int wave_lim = 32 * wave < nrows && before >= 0 ? before + last_row / p.g : -1;  // and its last
  const int seen = before >= 0 ? before + (it.row0 + nrows - 1) / p.g + 1 : 0;  // tokens the tile of rows sees
  const int all_see = before >= 0 ? before + it.row0 / p.g : -1;                // the last token that every row sees
  const int ntiles = p.num_blocks > 0 ? (seen + G::tokens - 1) / G::tokens : 0;
  const int tile0 = static_cast<int>(static_cast<int64_t>(ntiles) * split / p.nsplit);
  const int tile1 = static_cast<int>(static_cast<int64_t>(ntiles) * (split + 1) / p.nsplit);

  for (int i = tid; i < kBadKinds * D; i += kPfThreads) (&bad_dim[0][0])[i] = 0x7FFFFFFF;
  if (tid == 0) {
    bad_tok = p.num_blocks > 0 ? 0x7FFFFFFF : 0;
    any_bad = 0;
  }

  typedef typename std::conditional<G::f32, f32x4, uint4>::type Frag;
  // Query rows as the B operand.
  Frag q[G::ksteps];
  {
    const unsigned char* src = static_cast<const unsigned char*>(p.q) + orow * D * G::eb;
#pragma unroll
    for (int s = 0; s < G::ksteps; ++s)
      q[s] = active ? *reinterpret_cast<const Frag*>(src + (2 * s + half) * 16) : Frag{0, 0, 0, 0};
  }

  const size_t blk_stride = static_cast<size_t>(p.hkv) * C::blk_bytes;
  const unsigned char* kbase = static_cast<const unsigned char*>(p.k_cache) + static_cast<size_t>(kvh) * C::blk_bytes;
  const unsigned char* vbase = static_cast<const unsigned char*>(p.v_cache) + static_cast<size_t>(kvh) * C::blk_bytes;
  const int32_t* table = p.block_tables + static_cast<int64_t>(it.seq) * p.max_blocks;
  const int nblk = (seen + kTok - 1) / kTok;
  // Ids of the blocks that this wave's pieces of a tile come from, read through
  // the scalar cache (a vector load's wait would be one for the pieces in
  // flight too). Behind the last block: that one again. A block that is not in
  // the pool gives way to block 0: rows that see it are NaN, and to the others
  // its tokens are hidden ones.
  // (A vector value rather than an array, so that it stays in registers.)
  struct Ids {
    int id __attribute__((ext_vector_type(G::pieces)));
  };
  auto block_in_tile = [&](int i) { return (64 * wave + kPfThreads * i) / G::blk_pieces; };
  auto load_ids = [&](int tile) {
    Ids x;
#pragma unroll
    for (int i = 0; i < G::pieces; ++i) {
      const int lb = tile * G::blocks + block_in_tile(i);
      x.id[i] = scalar(table + (lb < nblk ? lb : nblk - 1));
    }
    return x;
  };
  auto check_ids = [&](Ids& x, int tile) {
#pragma unroll
    for (int i = 0; i < G::pieces; ++i)
      if (x.id[i] < 0 || x.id[i] >= p.num_blocks) {
        // (A tile behind the last repeats a block that was checked.)
        atomicMin(&bad_tok, (tile * G::blocks + block_in_tile(i)) * kTok);
        x.id[i] = 0;
      }
  };
  // fp8: the K scales times the softmax scale, and the V scales, of all of a
  // tile's blocks. A scale that is not finite makes every element of its block
  // infinite or NaN: rows that see the block are NaN, and the others must not
  // meet it (K scales: see the softmax).
  struct Scales {
    float k __attribute__((ext_vector_type(G::blocks)));
    float v __attribute__((ext_vector_type(G::blocks)));
  };
  struct AllIds {
    int id __attribute__((ext_vector_type(G::blocks)));
  };
  auto load_all_ids = [&](int tile) {
    AllIds x;
    if constexpr (KV == kKvFp8) {
#pragma unroll
      for (int i = 0; i < G::blocks; ++i) {
        const int lb = tile * G::blocks + i;
        x.id[i] = scalar(table + (lb < nblk ? lb : nblk - 1));
      }
    }
    return x;
  };
  auto load_scales = [&](const AllIds& x) {
    Scales s;
    if constexpr (KV == kKvFp8) {
#pragma unroll
      for (int i = 0; i < G::blocks; ++i) {
        const int id = x.id[i] < 0 || x.id[i] >= p.num_blocks ? 0 : x.id[i];
        s.k[i] = scalar(p.k_scale + id);
        s.v[i] = scalar(p.v_scale + id);
      }
    }
    return s;
  };
  auto check_scales = [&](Scales& s, int tile) {
    if constexpr (KV == kKvFp8) {
#pragma unroll
      for (int i = 0; i < G::blocks; ++i) {
        s.k[i] *= p.scale_log2;
        if (!(__builtin_fabsf(s.v[i]) < __builtin_inff())) {
          atomicMin(&bad_tok, tile * G::tokens + i * kTok);
          s.v[i] = 0.f;
        }
      }
    }
  };

  // A thread's pieces of a tile on their way from the cache.
  typedef typename G::Raw T;
  T kr[G::pieces], vr[G::pieces];
  uint32_t ks[KV == kKvMx4 ? G::pieces : 1];  // 4-bit caches: scale bytes
  uint2 vs[KV == kKvMx4 ? G::pieces : 1];
  auto load_k = [&](const Ids& x) {
#pragma unroll
    for (int i = 0; i < G::pieces; ++i) {
      const unsigned at = (tid + kPfThreads * i) % G::blk_pieces;
      const unsigned char* kb = kbase + static_cast<unsigned>(x.id[i]) * blk_stride;
      kr[i] = *reinterpret_cast<const T*>(kb + at * static_cast<unsigned>(sizeof(T)));
      if constexpr (KV == kKvMx4) ks[i] = kb[C::code_bytes + at * 8 / kMxGroup];
    }
  };
  auto load_v = [&](const Ids& x) {
#pragma unroll
    for (int i = 0; i < G::pieces; ++i) {
      const unsigned at = (tid + kPfThreads * i) % G::blk_pieces;
      const unsigned char* vb = vbase + static_cast<unsigned>(x.id[i]) * blk_stride;
      vr[i] = *reinterpret_cast<const T*>(vb + at * static_cast<unsigned>(sizeof(T)));
      if constexpr (KV == kKvMx4)
        vs[i] = *reinterpret_cast<const uint2*>(vb + C::code_bytes + at / G::vcols / kMxGroup * kTok + 8 * (at % G::vcols));
    }
  };
  auto kbuf = [&](int tile) { return lds + (tile & 1) * G::tensor_bytes; };
  auto vbuf = [&](int tile) { return lds + (2 + (tile & 1)) * G::tensor_bytes; };
  auto store_k = [&](int tile) {
#pragma unroll
    for (int i = 0; i < G::pieces; ++i) {
      const int piece = tid + kPfThreads * i, blk = piece / G::blk_pieces, at = piece % G::blk_pieces;
      uint4 x;
      if constexpr (KV == kKvMx4)
        x = mx4x8_to_bf16x8(kr[i], mx_scale<0>(ks[i]));
      else
        x = staged<KV>(kr[i]);
      *reinterpret_cast<uint4*>(kbuf(tile) + k_place<G>(blk * kTok + at / G::kcols, at % G::kcols)) = x;
    }
  };
  // Values past the last token seen are unused slots; those that some rows
  // see and others do not may be infinities or NaN, which a zero probability
  // would not keep out: they are taken out here and added, at the end, to the
  // rows that see them (whose probability of them counts as above 0, though it
  // may have underflowed).
  auto store_v = [&](int tile) {
    auto each = [&](auto hidden_c) {
#pragma unroll
      for (int i = 0; i < G::pieces; ++i) {
        const int piece = tid + kPfThreads * i, blk = piece / G::blk_pieces, at = piece % G::blk_pieces;
        const int dim = at / G::vcols, vcol = blk * G::vcols + at % G::vcols;
        uint4 x;
        if constexpr (KV == kKvMx4)
          x = mx4x8_to_bf16x8(vr[i], vs[i]);
        else
          x = staged<KV>(vr[i]);
        if constexpr (decltype(hidden_c)::value) {
          const int tok = tile * G::tokens + vcol * G::per;  // the piece's first token
          keep_first<G::f32>(x, seen - tok);
          if (any_nonfinite<G::f32>(x)) {
            drop_nonfinite<G::f32>(x, [&](int e, int kind) { atomicMin(&bad_dim[kind][dim], tok + e); });
            any_bad = 1;
          }
        }
        *reinterpret_cast<uint4*>(vbuf(tile) + v_place<G>(dim, vcol)) = x;
      }
    };
    if ((tile + 1) * G::tokens - 1 > all_see)
      each(std::true_type{});
    else
      each(std::false_type{});
  };

  f32x16 o[D / 32], s[G::tokens / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float ref = kNegInf, sum = 0.f;  // reference of the row (both halves alike), this lane's part of the sum
  uint4 pb[G::f32 ? 1 : G::vsteps];  // a tile's probabilities, the B operand of its value products

  auto scores = [&](int tile) {
#pragma unroll
    for (int t = 0; t < G::tokens / 32; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
      for (int j = 0; j < G::ksteps; ++j) {
        const Frag k = *reinterpret_cast<const Frag*>(kbuf(tile) + (t * G::ksteps + j) * 1024 + half * 512 +
                                                      ((ln ^ ((2 * j + half) & 15)) << 4));
        if constexpr (G::f32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[j][e], s[t], 0, 0, 0);
        } else {
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k),
                                                         __builtin_bit_cast(bf16x8, q[j]), s[t], 0, 0, 0);
        }
      }
    }
    reads_ahead<G::tokens / 32 * G::ksteps, G::f32 ? 4 : 1>();
  };
  auto softmax = [&](int tile, Scales& sc) {
    const int t0 = tile * G::tokens;
    if constexpr (KV == kKvFp8) {
      // What follows takes positive, finite scales; others are multiplied in
      // here. (An infinite one would turn the negative score of codes of both
      // signs, whose products with it have no sum, into no weight at all.)
      constexpr int kPosFinite = 0x080 | 0x100;  // positive: subnormal, normal
      bool positive = true;
#pragma unroll
      for (int b = 0; b < G::blocks; ++b) positive = positive && __builtin_amdgcn_classf(sc.k[b], kPosFinite);
      if (!positive) {
        asm volatile("");
#pragma unroll
        for (int b = 0; b < G::blocks; ++b)
          if (!(__builtin_fabsf(sc.k[b]) < __builtin_inff())) atomicMin(&bad_tok, t0 + b * kTok);
#pragma unroll
        for (int t = 0; t < G::tokens / 32; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[t][i] *= sc.k[(32 * t + reg_token<G::f32>(i)) / kTok];
#pragma unroll
        for (int b = 0; b < G::blocks; ++b) sc.k[b] = 1.f;
      }
    }
    // Hidden tokens: -inf. (The empty asm keeps this a branch: as selects it
    // would cost every tile two instructions per score.)
    if (t0 + G::tokens - 1 > first_lim) {
      asm volatile("");
      const int left = lim - t0 - half * (G::f32 ? 4 : 8);
#pragma unroll
      for (int t = 0; t < G::tokens / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = 32 * t + reg_token<G::f32>(i) <= left ? s[t][i] : kNegInf;
    }
    float mx = kNegInf;
    if constexpr (KV == kKvFp8) {
#pragma unroll
      for (int b = 0; b < G::blocks; ++b) {
        float m = s[b / 2][8 * (b & 1)];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = fmaxf(m, s[b / 2][8 * (b & 1) + i]);
        mx = fmaxf(mx, m * sc.k[b]);
      }
      mx = halves_max(mx);
    } else {
#pragma unroll
      for (int t = 0; t < G::tokens / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
      mx = halves_max(mx) * p.scale_log2;  // (the scale is positive)
    }
    if (__builtin_amdgcn_ballot_w64(mx > ref + kRefSlack || (ref == kNegInf && mx > kNegInf)) != 0) {
      const float now = mx > ref ? mx : ref;
      const float f = ref == kNegInf ? 0.f : __builtin_amdgcn_exp2f(ref - now);
      sum *= f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] *= f;
      ref = now;
    }
    const float sub = ref == kNegInf ? 0.f : ref;
#pragma unroll
    for (int t = 0; t < G::tokens / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float f = KV == kKvFp8 ? sc.k[(32 * t + reg_token<G::f32>(i)) / kTok] : p.scale_log2;
        s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], f, -sub));
        if constexpr (G::f32 || KV == kKvFp8) sum += s[t][i];
      }
    if constexpr (!G::f32) {
#pragma unroll
      for (int j = 0; j < G::vsteps; ++j) {
        float pv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          pv[e] = s[j >> 1][8 * (j & 1) + e];
          if constexpr (KV == kKvFp8) pv[e] *= sc.v[j];
        }
        pb[j] = uint4{pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]), pack_bf16x2(pv[4], pv[5]),
                      pack_bf16x2(pv[6], pv[7])};
        // The sum of the rounded probabilities, which the product uses (fp8:
        // those are multiplied by the V scales).
        if constexpr (KV != kKvFp8) {
          const uint32_t w[4] = {pb[j].x, pb[j].y, pb[j].z, pb[j].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) sum = add_bf16x2(w[e], sum);
        }
      }
    }
  };
  auto values = [&](int tile) {
#pragma unroll
    for (int j = 0; j < G::vsteps; ++j)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const Frag v = *reinterpret_cast<const Frag*>(vbuf(tile) + (d * G::vsteps + j) * 1024 + half * 512 +
                                                      ((ln ^ (((2 * j + half) & (G::vcols - 1)) * (16 / G::vcols))) << 4));
        if constexpr (G::f32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], s[0][4 * j + e], o[d], 0, 0, 0);
        } else {
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pb[j]),
                                                         o[d], 0, 0, 0);
        }
      }
    reads_ahead<G::vsteps * D / 32, G::f32 ? 4 : 1>();
  };

  if (tile0 < tile1) {
    __syncthreads();  // bad_dim and bad_tok are set
    AllIds all = load_all_ids(tile0);
    Ids ids = load_ids(tile0), next = load_ids(tile0 + 1);
    check_ids(ids, tile0);
    load_k(ids);
    load_v(ids);
    Scales sc = load_scales(all), sc_next;
    all = load_all_ids(tile0 + 1);
    store_k(tile0);
    store_v(tile0);
    check_ids(next, tile0 + 1);
    load_k(next);
    load_v(next);
    next = load_ids(tile0 + 2);
    __syncthreads();
    for (int tile = tile0; tile < tile1; ++tile) {
      sc_next = load_scales(all);
      all = load_all_ids(tile + 2);
      check_scales(sc, tile);
      if (tile * G::tokens <= wave_lim) {
        scores(tile);
        softmax(tile, sc);
        values(tile);
      }
      sc = sc_next;
      if (tile + 1 < tile1) {
        store_k(tile + 1);
        store_v(tile + 1);
        check_ids(next, tile + 2);
        load_k(next);
        load_v(next);
        next = load_ids(tile + 3);
      }
      __syncthreads();
    }
  }
  __syncthreads();  // bad_dim and bad_tok are whole
  if (!active) return;
  const int first_bad = bad_tok;
  const bool add_bad = any_bad != 0;

  sum += __shfl_xor(sum, 32);
  const float qnan = __builtin_nanf("");
  const bool nan_row = bad || lim >= first_bad;
  if (nan_row) sum = qnan;
  // Lane (row, half): dims 32 d + 8 i + 4 half .. + 4.
  const float f = p.nsplit > 1 ? 1.f : (nan_row ? qnan : (sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : qnan)));
  const int64_t part_row = static_cast<int64_t>(split) * p.num_tokens * p.hq + orow;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dim = 32 * d + 8 * i + 4 * half;
      f32x4 x = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      x *= f;
      if (add_bad) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (lim >= bad_dim[kBadPos][dim + e]) x[e] += __builtin_inff();
          if (lim >= bad_dim[kBadNeg][dim + e]) x[e] -= __builtin_inff();
          if (lim >= bad_dim[kBadNan][dim + e]) x[e] = qnan;
        }
      }
      if (p.nsplit > 1)
        *reinterpret_cast<f32x4*>(p.part_o + part_row * D + dim) = x;
      else
        store_out4(p.out, p.out_bf16 != 0, orow * D + dim, x);
    }
  if (p.nsplit > 1 && half == 0)
    *reinterpret_cast<f32x2*>(p.part_ml + 2 * part_row) = f32x2{ref, sum};
}

// The splits of a row joined, in their order. A wave per row; lane j holds
// split j's reference and sum (at most kPrefillMaxSplit of them). Rows
// behind the last sequence are left as they are.
template <int D>
__global__ __launch_bounds__(256) void prefill_merge_kernel(PrefillParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t r = p.unit0 + static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t rows = static_cast<int64_t>(p.num_tokens) * p.hq;
  if (r >= rows || r / p.hq < p.tok_offsets[0] || r / p.hq >= p.tok_offsets[p.num_seqs]) return;
  f32x2 ml = {kNegInf, 0.f};
  if (lane < p.nsplit) ml = *reinterpret_cast<const f32x2*>(p.part_ml + 2 * (lane * rows + r));
  const bool nan = __builtin_amdgcn_ballot_w64(ml.y != ml.y) != 0;
  float mx = ml.x;
#pragma unroll
  for (int o = 1; o < kPrefillMaxSplit; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  const float w = ml.x == kNegInf ? 0.f : __builtin_amdgcn_exp2f(ml.x - mx);
  float den = ml.y * w;
#pragma unroll
  for (int o = 1; o < kPrefillMaxSplit; o <<= 1) den += __shfl_xor(den, o);
  constexpr int kEl = D / 64;
  float acc[kEl] = {};
  for (int k = 0; k < p.nsplit; ++k) {
    const float wk = __shfl(w, k);
#pragma unroll
    for (int e = 0; e < kEl; ++e) acc[e] += wk * p.part_o[(k * rows + r) * D + kEl * lane + e];
  }
  den = __shfl(den, 0);
  const float inv = nan ? __builtin_nanf("") : (den > 0.f ? 1.f / den : 0.f);
#pragma unroll
  for (int e = 0; e < kEl; ++e) {
    const int64_t at = r * D + kEl * lane + e;
    const float x = acc[e] * inv;
    if (p.out_bf16)
      static_cast<uint16_t*>(p.out)[at] = static_cast<uint16_t>(pack_bf16x2(x, x));
    else
      static_cast<float*>(p.out)[at] = x;
  }
}

template <int D, int KV>
hipError_t launch_prefill_t(PrefillParams p, hipStream_t stream) {
  // (A launch holds fewer than 2^32 threads.)
  constexpr int64_t kMost = 0xFFFFFFFFll / kPfThreads;
  p.units = prefill_items(p.num_seqs, p.num_tokens, p.g) * p.hkv * p.nsplit;
  for (p.unit0 = 0; p.unit0 < p.units; p.unit0 += kMost) {
    const int64_t n = p.units - p.unit0 < kMost ? p.units - p.unit0 : kMost;
    hipLaunchKernelGGL((prefill_kernel<D, KV>), dim3(static_cast<unsigned>(n)), dim3(kPfThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.nsplit > 1) {
    const int64_t rows = static_cast<int64_t>(p.num_tokens) * p.hq;
    constexpr int64_t kMostRows = 0xFFFFFFFFll / 256 * 4;
    for (p.unit0 = 0; p.unit0 < rows; p.unit0 += kMostRows) {
      const int64_t n = rows - p.unit0 < kMostRows ? rows - p.unit0 : kMostRows;
      hipLaunchKernelGGL((prefill_merge_kernel<D>), dim3(static_cast<unsigned>((n + 3) / 4)), dim3(256), 0, stream, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

template <int D>
hipError_t launch_prefill_d(const PrefillParams& p, int kv_kind, hipStream_t stream) {
  switch (kv_kind) {
    case kKvF32: return launch_prefill_t<D, kKvF32>(p, stream);
    case kKvBf16: return launch_prefill_t<D, kKvBf16>(p, stream);
    case kKvFp8: return launch_prefill_t<D, kKvFp8>(p, stream);
    default: return launch_prefill_t<D, kKvMx4>(p, stream);
  }
}

}  // namespace

hipError_t launch_prefill(const PrefillParams& p, int head_dim, int kv_kind, hipStream_t stream) {
  return head_dim == 128 ? launch_prefill_d<128>(p, kv_kind, stream) : launch_prefill_d<64>(p, kv_kind, stream);
}

}  // namespace tts
