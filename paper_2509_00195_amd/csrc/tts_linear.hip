// Products with trained weights, and the norm before them.
//
// out[m][n] = act(sum_k x[m][k] w[n][k] + bias[n]) + residual[m][n], and the
// gated form act(gate) * up of two such sums. Both operands have the inner
// dimension contiguous. The weights are the matrix instructions' first
// operand and x the second, so that a lane ends with four consecutive columns
// of one row of the output. All of it is done in pieces of 16 bytes (8 bf16
// values, one 16x16x32 instruction; 4 fp32 values, four 16x16x4 ones): which
// value of a step lies in which lane group does not matter as long as both
// operands agree. Sums are fp32, the result is rounded once.
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "tts_device.h"
#include "tts_linear.h"

namespace tts {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Loads and stores at the addresses of a caller's rows, which need only the
// alignment of an element (the hardware takes them, an instruction each).
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

template <typename E>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (sizeof(E) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
    return c;
  }
}

// 16 bytes of a row of `end` bytes from byte `at`; what lies behind the end is zero and is not read.
template <typename E>
__device__ __forceinline__ u32x4 load_piece(const char* row, int at, int end) {
  if (at + 16 <= end) return *reinterpret_cast<const u32x4u*>(row + at);
  u32x4 r = {0u, 0u, 0u, 0u};
  if constexpr (sizeof(E) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + 2 * i < end)
        r[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(row + at + 2 * i)) << (16 * (i % 2));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 4 * i < end) r[i] = *reinterpret_cast<const uint32_t*>(row + at + 4 * i);
  }
  return r;
}

__device__ __forceinline__ float activate(float y, int act) {
  switch (act) {
    case kActRelu: return y < 0.f ? 0.f : y;  // (NaN stays)
    case kActSilu: return y / (1.f + __expf(-y));
    case kActGelu: return 0.5f * y * erfcf(-0.70710678118654752f * y);
    case kActGeluTanh: {  // 1 + tanh z = 2 / (1 + exp(-2 z))
      const float z = 0.79788456080286536f * (y + 0.044715f * y * y * y);
      return y / (1.f + __expf(-2.f * z));
    }
    default: return y;
  }
}

// `count` (at most 4) values from element i of an array of bf16 or fp32.
__device__ __forceinline__ f32x4 load_row4(const void* p, int64_t i, int count, bool is_bf16) {
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  if (is_bf16) {
    const __bf16* s = static_cast<const __bf16*>(p) + i;
    if (count == 4) return __builtin_convertvector(*reinterpret_cast<const bf16x4u*>(s), f32x4);
    for (int j = 0; j < 3; ++j)
      if (j < count) r[j] = static_cast<float>(s[j]);
  } else {
    const float* s = static_cast<const float*>(p) + i;
    if (count == 4) return *reinterpret_cast<const f32x4u*>(s);
    for (int j = 0; j < 3; ++j)
      if (j < count) r[j] = s[j];
  }
  return r;
}

__device__ __forceinline__ int columns(const LinearParams& p, int n) { return p.n - n < 4 ? p.n - n : 4; }

__device__ __forceinline__ int least(int a, int b) { return a < b ? a : b; }

// What an output's four columns are made with beside their sums, four values
// each: bits as they are stored, where every row has whole quads of columns,
// else fp32. Loaded early, and with no branch but uniform ones: where lanes
// branch, the compiler waits for each load before the next (a wave's residual
// in a 256 x 256 tile was 32 round trips one after another: 8192 x 3584 x 3584
// with all of it from memory 216 -> 184 us).
typedef u32x4 Four;

struct FourType {
  bool wide, is_bf16;  // whole quads, and their type

  __device__ __forceinline__ Four load(const void* p, int64_t i) const {  // wide
    if (!is_bf16) return *reinterpret_cast<const u32x4u*>(static_cast<const float*>(p) + i);
    const u32x2 r = *reinterpret_cast<const u32x2u*>(static_cast<const uint16_t*>(p) + i);
    return Four{r[0], r[1], 0u, 0u};
  }
  __device__ __forceinline__ f32x4 value(Four v) const {
    if (!wide || !is_bf16) return __builtin_bit_cast(f32x4, v);
    const uint32_t b[4] = {v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u};
    return f32x4{__builtin_bit_cast(float, b[0]), __builtin_bit_cast(float, b[1]), __builtin_bit_cast(float, b[2]),
                 __builtin_bit_cast(float, b[3])};
  }
};

__device__ __forceinline__ FourType bias_type(const LinearParams& p) { return {p.n % 4 == 0, p.in_bf16 != 0}; }
__device__ __forceinline__ FourType residual_type(const LinearParams& p) { return {p.n % 4 == 0, p.out_bf16 != 0}; }

// Of N places (m(i), n(i)); behind the last row or column what is loaded is not used.
template <int N, typename F>
__device__ __forceinline__ void load_bias(const LinearParams& p, int plane, Four (&r)[N], F n) {
  const FourType t = bias_type(p);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = Four{0u, 0u, 0u, 0u};
  if (!p.bias[plane]) return;
  if (t.wide) {
    if (t.is_bf16)
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = FourType{true, true}.load(p.bias[plane], least(n(i), p.n - 4));
    else
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = FourType{true, false}.load(p.bias[plane], least(n(i), p.n - 4));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (n(i) < p.n) r[i] = __builtin_bit_cast(Four, load_row4(p.bias[plane], n(i), columns(p, n(i)), t.is_bf16));
  }
}

template <int N, typename M, typename F>
__device__ __forceinline__ void load_residual(const LinearParams& p, Four (&r)[N], M m, F n) {
  const FourType t = residual_type(p);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = Four{0u, 0u, 0u, 0u};
  if (!p.residual) return;
  const auto at = [&](int i) { return least(m(i), p.rows - 1) * p.residual_stride + least(n(i), p.n - 4); };
  if (t.wide) {
    if (t.is_bf16)
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = FourType{true, true}.load(p.residual, at(i));
    else
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = FourType{true, false}.load(p.residual, at(i));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (m(i) < p.rows && n(i) < p.n)
        r[i] = __builtin_bit_cast(Four, load_row4(p.residual, m(i) * p.residual_stride + n(i), columns(p, n(i)), t.is_bf16));
  }
}

// act(y + bias), gated: times (up + its bias).
template <bool GATED>
__device__ __forceinline__ f32x4 activated(const LinearParams& p, f32x4 bias, f32x4 up_bias, f32x4 y, f32x4 up) {
  y += bias;
  if (p.act != kActNone)
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = activate(y[j], p.act);
  if constexpr (GATED) y *= up + up_bias;
  return y;
}

__device__ __forceinline__ void store_out(const LinearParams& p, int m, int n, f32x4 y) {
  const int count = columns(p, n);
  const int64_t at = m * p.out_stride + n;
  if (p.out_bf16) {
    __bf16* o = static_cast<__bf16*>(p.out) + at;
    const bf16x4 r = __builtin_convertvector(y, bf16x4);
    if (count == 4)
      *reinterpret_cast<bf16x4u*>(o) = r;
    else
      for (int j = 0; j < 3; ++j)
        if (j < count) o[j] = r[j];
  } else {
    float* o = static_cast<float*>(p.out) + at;
    if (count == 4)
      *reinterpret_cast<f32x4u*>(o) = y;
    else
      for (int j = 0; j < 3; ++j)
        if (j < count) o[j] = y[j];
  }
}

// Partial sums of a split, columns n .. n + 3 of row m of plane 0 (gate) or 1 (up).
__device__ __forceinline__ int64_t part_at(const LinearParams& p, int split, int plane, int planes, int m, int n) {
  return ((static_cast<int64_t>(split) * planes + plane) * p.rows + m) * p.n + n;
}

__device__ __forceinline__ void store_part(float* dst, int count, f32x4 y) {
  if (count == 4)
    *reinterpret_cast<f32x4u*>(dst) = y;
  else
    for (int j = 0; j < 3; ++j)
      if (j < count) dst[j] = y[j];
}

template <bool GATED>
__device__ __forceinline__ void store_parts(const LinearParams& p, int split, int m, int n, f32x4 y, f32x4 up) {
  constexpr int kPlanes = GATED ? 2 : 1;
  store_part(p.part + part_at(p, split, 0, kPlanes, m, n), columns(p, n), y);
  if constexpr (GATED) store_part(p.part + part_at(p, split, 1, kPlanes, m, n), columns(p, n), up);
}

// ---- loads into LDS ------------------------------------------------------------

constexpr uint32_t kOutside = 0x80000000u;  // behind the end of every tile's buffer: reads as zero

// A buffer whose loads are checked against its size, and its loads into LDS (16
// bytes to a lane, lane after lane from `lds`). The builtins are known to the
// device's compilation alone.
struct Rows {
#if defined(__HIP_DEVICE_COMPILE__)
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ void set(const char* base, uint32_t bytes) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00020000);
  }
  __device__ __forceinline__ void load(char* lds, uint32_t offset, int at) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)lds, 16, offset, at, 0, 0);
  }
#else
  __device__ void set(const char*, uint32_t) {}
  __device__ void load(char*, uint32_t, int) const {}
#endif
};

// Waits for this wave's loads into LDS, but for the newest N: a barrier behind
// it then means that all waves' have landed (the barrier alone waits for none).
template <int N = 0>
__device__ __forceinline__ void landed() {
  static_assert(N < 64, "the counter's width");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);  // vmcnt(N)
  __builtin_amdgcn_sched_barrier(0);
}

// A barrier that waits for no load in flight (__syncthreads waits for all).
// What a wave has read from LDS before it must have been used: the reads are
// then over. The empty statements keep the compiler from moving memory
// accesses across.
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// What a wave's lanes have written to LDS is read by its other lanes behind
// this: a wave's accesses to LDS are made in their order, so that only the
// compiler has to keep it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f(integral_constant<int, 0>{}), ..., f(integral_constant<int, N - 1>{}).
template <typename F, int... J>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, J...>) {
  (f(std::integral_constant<int, J>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each(f, std::make_integer_sequence<int, N>{});
}

// Whether f(integral_constant<int, 0>{}), ... are all true; ends with the first that is not.
template <typename F, int... J>
__device__ __forceinline__ bool all(F f, std::integer_sequence<int, J...>) {
  return (f(std::integral_constant<int, J>{}) && ...);
}
template <int N, typename F>
__device__ __forceinline__ bool all(F f) {
  return all(f, std::make_integer_sequence<int, N>{});
}

// (One value to the wave, which the compiler then keeps in a scalar register.)
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / 64); }

// Place of a workgroup in the order of the tiles (those of the first split,
// then of the next): workgroups go to the eight XCDs in turn, and this gives
// each a run of consecutive tiles, whose shared rows its L2 then serves.
__device__ __forceinline__ int place_of(int id, int places) {
  const int per = places / 8, rest = places % 8, xcd = id % 8;
  return xcd * per + (xcd < rest ? xcd : rest) + id / 8;
}

// ---- small tiles ---------------------------------------------------------------

constexpr int kThinWaves = kThinThreads / 64;
constexpr int kThinRow = kThinChunk;  // bytes of a row to a stage: a quarter to each wave

// Few rows: bound by the weights' bytes and, where many workgroups read the
// same rows of x, by what a compute unit draws from its L2 (some 50 bytes a
// cycle). Tiles of BM rows of x and BN rows of weights (gated: half gate, half
// up, of the same columns) pass through S stages in LDS, S - 1 of them in
// flight, each row 256 bytes long to a stage in 16 pieces of 16, piece c of row
// r at c ^ (r & 15): the permutation leaves no bank conflict. Every wave
// multiplies the whole tile over its quarter of a stage's inner dimension, so
// that each byte is read from LDS once; the waves' sums are added at the end,
// in their order. Measured (bf16): 1 x 1536 x 2048 4.4 us and 16 x 1536 x 6144
// gated 9.0 (launches 3.5), 64 x 3584 x 4608 11.2, of which 33 MB of weights are
// 6.6 at a copy's rate: 192 workgroups of 32 x 48, each of which draws 0.57 MB.
// Rows of 64 bytes to a stage, for more stages, were slower.
template <typename E, int BM, int BN, int S, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(kThinThreads) void thin_kernel(LinearParams p) {
  constexpr int TM = BM / 16, TN = BN / 16, kPlanes = GATED ? 2 : 1, kCols = BN / kPlanes;
  constexpr int kStage = (BM + BN) * kThinRow, kLoads = TM + TN;
  static_assert(S >= 2 && S <= 8 && (ALIGNED || S == 2) && kLoads * (S - 2) < 64, "stages");
  __shared__ __attribute__((aligned(16))) char s0[kStage], s1[kStage], s2[S > 2 ? kStage : 16], s3[S > 3 ? kStage : 16],
      s4[S > 4 ? kStage : 16], s5[S > 5 ? kStage : 16], s6[S > 6 ? kStage : 16], s7[S > 7 ? kStage : 16];
  // (An array each, not one: the compiler then knows which of them a load writes.)
  const auto stage = [&](auto i) -> char* {
    constexpr int k = decltype(i)::value % S;
    if constexpr (k == 0) return s0;
    else if constexpr (k == 1) return s1;
    else if constexpr (k == 2) return s2;
    else if constexpr (k == 3) return s3;
    else if constexpr (k == 4) return s4;
    else if constexpr (k == 5) return s5;
    else if constexpr (k == 6) return s6;
    else return s7;
  };
  const int wave = wave_id(), lane = static_cast<int>(threadIdx.x) % 64;
  const int tiles = p.m_tiles * p.n_tiles, place = place_of(static_cast<int>(blockIdx.x), tiles * p.splits);
  const int id = place % tiles, split = place / tiles;
  const int m0 = id % p.m_tiles * BM, n0 = id / p.m_tiles * kCols;
  const int total = (p.k_bytes + kThinRow - 1) / kThinRow;
  const int first = split * p.chunks, end = first + p.chunks < total ? first + p.chunks : total;
  const int stop = end == total ? p.k_bytes : end * kThinRow;

  // A load takes four rows to a wave, sixteen to the workgroup.
  const int sub = wave * 4 + (lane >> 4), piece = (lane & 15) ^ sub;
  const int rows_m = least(p.rows - m0, BM), rows_n = least(p.n - n0, kCols);
  const char* xb = static_cast<const char*>(p.x) + m0 * p.x_stride;
  const char* wb[kPlanes];
  Rows xr, wr[kPlanes];
  xr.set(xb, static_cast<uint32_t>((rows_m - 1) * p.x_stride + p.k_bytes));
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) {
    wb[i] = static_cast<const char*>(p.w[i]) + n0 * p.w_stride;
    wr[i].set(wb[i], static_cast<uint32_t>((rows_n - 1) * p.w_stride + p.k_bytes));
  }
  const uint32_t off_n = static_cast<uint32_t>(sub * p.w_stride + 16 * piece);
  const uint32_t off_m = static_cast<uint32_t>(sub * p.x_stride + 16 * piece);
  constexpr int kTilesN = TN / kPlanes;  // of a plane
  u32x4 held[ALIGNED ? 1 : kLoads];

  // Chunk c into a stage (not aligned: into registers, for put()).
  const auto start = [&](char* to, int c) {
    const int at = c * kThinRow;
    if constexpr (ALIGNED) {
      const bool out = at + 16 * piece >= stop;
      const uint32_t from_n = out ? kOutside : off_n, from_m = out ? kOutside : off_m;
      const uint32_t step_n = static_cast<uint32_t>(16 * p.w_stride), step_m = static_cast<uint32_t>(16 * p.x_stride);
#pragma unroll
      for (int i = 0; i < TN; ++i)
        wr[i / kTilesN].load(to + (i * 16 + wave * 4) * kThinRow, from_n + (i % kTilesN) * step_n, at);
#pragma unroll
      for (int i = 0; i < TM; ++i) xr.load(to + (BN + i * 16 + wave * 4) * kThinRow, from_m + i * step_m, at);
    } else {
      const auto fetch = [&](auto whole) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const bool is_x = i >= TN;
          const int row = is_x ? least((i - TN) * 16 + sub, rows_m - 1) : least(i % kTilesN * 16 + sub, rows_n - 1);
          const char* src = is_x ? xb + row * p.x_stride : wb[is_x ? 0 : i / kTilesN] + row * p.w_stride;
          if constexpr (whole.value)
            held[i] = *reinterpret_cast<const u32x4u*>(src + at + 16 * piece);
          else
            held[i] = load_piece<E>(src, at + 16 * piece, stop);
        }
      };
      if (at + kThinRow <= stop)
        fetch(std::true_type{});
      else
        fetch(std::false_type{});
    }
  };
  const auto put = [&](char* to) {
#pragma unroll
    for (int i = 0; i < (ALIGNED ? 0 : kLoads); ++i)
      *reinterpret_cast<u32x4*>(to + (i * 16 + wave * 4) * kThinRow + lane * 16) = held[i];
  };

  const int row = lane & 15, group = lane >> 4;
  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int from = row * kThinRow + ((4 * wave + group) ^ row) * 16;
  const auto multiply = [&](const char* at) {
    u32x4 a[TN], b[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) a[i] = *reinterpret_cast<const u32x4*>(at + from + i * 16 * kThinRow);
#pragma unroll
    for (int j = 0; j < TM; ++j) b[j] = *reinterpret_cast<const u32x4*>(at + from + (BN + j * 16) * kThinRow);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = mma<E>(a[i], b[j], acc[i][j]);
  };

  // A thread's outputs, and what they are made with (older than the chunks'
  // loads, so that waiting for these covers it).
  constexpr int kQuads = kCols / 4, kItems = BM * kQuads, kEach = (kItems + kThinThreads - 1) / kThinThreads;
  const auto m_of = [&](int e) { return m0 + (static_cast<int>(threadIdx.x) + e * kThinThreads) / kQuads; };
  const auto n_of = [&](int e) { return n0 + (static_cast<int>(threadIdx.x) + e * kThinThreads) % kQuads * 4; };
  Four bias[kPlanes][kEach], residual[kEach];
  if (p.splits == 1) {
#pragma unroll
    for (int i = 0; i < kPlanes; ++i) load_bias(p, i, bias[i], n_of);
    load_residual(p, residual, m_of, n_of);
  }
  __builtin_amdgcn_sched_barrier(0);

  // Stage j's chunk has landed once all but the S - 2 newer ones have; behind
  // the barrier the stage read before it is free for the chunk S - 1 further
  // on. Chunks behind the end load nothing and are zero.
  if constexpr (ALIGNED) {
    each<S - 1>([&](auto j) { start(stage(j), first + decltype(j)::value); });
  } else {
    start(s0, first);
  }
  const auto step = [&](auto j, int c) {
    constexpr int k = decltype(j)::value;
    if constexpr (ALIGNED) {
      landed<kLoads*(S - 2)>();
      barrier();
    } else {
      put(stage(j));
      __syncthreads();
    }
    start(stage(std::integral_constant<int, k + S - 1>{}), c + (ALIGNED ? S - 1 : 1));
    __builtin_amdgcn_sched_barrier(0);
    multiply(stage(j));
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int c = first; c < end; c += S)
    each<S>([&](auto j) { step(j, c + decltype(j)::value); });

  // The waves' sums, [wave][tile][lane], then whole runs of columns.
  static_assert(kThinWaves * TN * TM * 1024 <= S * kStage, "the sums' place");
  landed();
  __syncthreads();
  constexpr int kSums = kStage / 1024;  // tiles of sums to a stage
  const auto sum_at = [&](int i) {  // (wave * tiles + tile)
    const int k = i / kSums;
    char* at = k == 0 ? s0 : k == 1 ? s1 : k == 2 ? s2 : s3;
    return reinterpret_cast<f32x4*>(at + i % kSums * 1024);
  };
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) sum_at(wave * TN * TM + i * TM + j)[lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = static_cast<int>(threadIdx.x) + e * kThinThreads, r = i / kQuads, q = i % kQuads;
    const int m = m0 + r, n = n0 + 4 * q;
    if ((kItems % kThinThreads != 0 && i >= kItems) || m >= p.rows || n >= p.n) continue;
    const int l = (r & 15) + 16 * (q & 3), t = q / 4 * TM + r / 16;
    f32x4 y = sum_at(t)[l], up = y;
#pragma unroll
    for (int w = 1; w < kThinWaves; ++w) y += sum_at(w * TN * TM + t)[l];
    if constexpr (GATED) {
      up = sum_at(t + kTilesN * TM)[l];
#pragma unroll
      for (int w = 1; w < kThinWaves; ++w) up += sum_at(w * TN * TM + t + kTilesN * TM)[l];
    }
    if (p.splits > 1)
      store_parts<GATED>(p, split, m, n, y, up);
    else
      store_out(p, m, n, activated<GATED>(p, bias_type(p).value(bias[0][e]), bias_type(p).value(bias[kPlanes - 1][e]), y, up) +
                             residual_type(p).value(residual[e]));
  }
}

// ---- tiles -------------------------------------------------------------------

// Many rows: BM rows of x by BN rows of weights to a workgroup of WM x WN
// waves, whose sums stay in registers, with SM and SN stages of the operands in
// LDS. Bound on long calls by the matrix instructions, at a clock that falls to
// 1.84 GHz under them, and by the waits at a chunk's barrier: the matrix cores
// are busy 0.63 of the time, the waves wait 0.32 of theirs. In smaller calls
// bound by the bytes that a unit draws from its L2, which a larger tile halves.
// Measured (bf16): 8192 x 3584 x 28672 (gated, 256 x 256) 1,285 us or 1,310
// TFLOP/s, a large product of the library 1,290 to 1,560; 8192 x 3584 x 3584 182
// us with a residual from memory, where 448 tiles take two rounds of 256 units;
// 320 x 14336 x 3584 (128 x 256 in six parts) 52 in all, 7 of them for joining
// the parts; 64 x 3584 x 14336 gated (64 x 128) 43, its weights 41 at a copy's
// rate. Weights have a third stage beside x's two in the largest tile, all that
// LDS holds: a load that comes late then stops nothing. Instructions of 32 x 32
// x 16 were slower (1,388 us against 1,350), so was a tile for four waves of
// 128 x 128 (the compiler spills: it lets the sums' registers change).
//
// A tile's rows lie in LDS 128 bytes each, in eight pieces of 16 whose places
// are permuted by the row (piece c of row r at c ^ (r & 7)), so that the same
// piece of 16 rows, which a matrix operand reads, is spread over the banks (no
// conflict is counted). The LDS side of a load into LDS is fixed (lane after
// lane), so the lanes' global addresses carry the permutation.
template <typename E, int BM, int BN, int WM, int WN, int SM, int SN, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN, 2) void tile_kernel(LinearParams p) {
  constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 tiles of a wave
  constexpr int kLoadsN = BN / 8 / kWaves, kLoadsM = BM / 8 / kWaves, kLoads = kLoadsN + kLoadsM;
  constexpr int kPlanes = GATED ? 2 : 1;
  constexpr int kCols = BN / kPlanes;
  static_assert(SM >= 2 && SM <= SN && SN <= SM + 1 && SN <= 4 && (ALIGNED || SN == 2), "stages");
  constexpr int kBytesN = BN * kLinearChunk, kBytesM = BM * kLinearChunk;
  __shared__ __attribute__((aligned(16))) char n_0[kBytesN], n_1[kBytesN], n_2[SN > 2 ? kBytesN : 16],
      n_3[SN > 3 ? kBytesN : 16], m_0[kBytesM], m_1[kBytesM], m_2[SM > 2 ? kBytesM : 16], m_3[SM > 3 ? kBytesM : 16];
  const auto stage_n = [&](auto i) -> char* {
    constexpr int k = decltype(i)::value % SN;
    if constexpr (k == 0) return n_0;
    else if constexpr (k == 1) return n_1;
    else if constexpr (k == 2) return n_2;
    else return n_3;
  };
  const auto stage_m = [&](auto i) -> char* {
    constexpr int k = decltype(i)::value % SM;
    if constexpr (k == 0) return m_0;
    else if constexpr (k == 1) return m_1;
    else if constexpr (k == 2) return m_2;
    else return m_3;
  };
  const int wave = wave_id(), lane = static_cast<int>(threadIdx.x) % 64;

  // Tiles in groups of 8 along x's rows.
  const int tiles = p.m_tiles * p.n_tiles, spot = place_of(static_cast<int>(blockIdx.x), tiles * p.splits);
  const int id = spot % tiles, split = spot / tiles;
  constexpr int kGroup = 8;
  const int in_group = kGroup * p.n_tiles, g0 = id / in_group * kGroup;
  const int height = p.m_tiles - g0 < kGroup ? p.m_tiles - g0 : kGroup;
  const int m0 = (g0 + id % in_group % height) * BM, n0 = id % in_group / height * kCols;

  const int total = (p.k_bytes + kLinearChunk - 1) / kLinearChunk;
  const int first = split * p.chunks, end = first + p.chunks < total ? first + p.chunks : total;
  const int stop = end == total ? p.k_bytes : end * kLinearChunk;  // of a row's bytes

  const int sub = lane >> 3, piece = (lane & 7) ^ sub;  // a load's 8 rows: this lane's row and piece of it
  const int rows_m = p.rows - m0 < BM ? p.rows - m0 : BM, rows_n = p.n - n0 < kCols ? p.n - n0 : kCols;
  const char* xb = static_cast<const char*>(p.x) + m0 * p.x_stride;
  const char* wb[kPlanes];
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) wb[i] = static_cast<const char*>(p.w[i]) + n0 * p.w_stride;

  // Rows of load i, within the operand (gated: within its plane).
  constexpr int kStep = 8 * kWaves;
  const auto row_n = [&](int i) { return (i % (kLoadsN / kPlanes)) * kStep + wave * 8 + sub; };
  const auto row_m = [&](int i) { return i * kStep + wave * 8 + sub; };

  // (Rows behind the last one start behind the buffer's end.)
  Rows xr, wr[kPlanes];
  xr.set(xb, static_cast<uint32_t>((rows_m - 1) * p.x_stride + p.k_bytes));
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) wr[i].set(wb[i], static_cast<uint32_t>((rows_n - 1) * p.w_stride + p.k_bytes));
  const uint32_t off_n = static_cast<uint32_t>(row_n(0) * p.w_stride + 16 * piece);
  const uint32_t off_m = static_cast<uint32_t>(row_m(0) * p.x_stride + 16 * piece);
  u32x4 held[ALIGNED ? 1 : kLoadsN + kLoadsM];

  // Load i of chunk c of the weights and of x (aligned: into LDS; else into registers, for put()).
  constexpr int kLoadsPlane = kLoadsN / kPlanes;
  const uint32_t step_n = static_cast<uint32_t>(kStep * p.w_stride), step_m = static_cast<uint32_t>(kStep * p.x_stride);
  const auto fetch = [&](const char* src, int at) -> u32x4 {
    if (at + kLinearChunk <= stop) return *reinterpret_cast<const u32x4u*>(src + at + 16 * piece);
    return load_piece<E>(src, at + 16 * piece, stop);
  };
  const auto load_n = [&](char* stage, int c, int i) {
    const int at = c * kLinearChunk;
    if constexpr (ALIGNED)
      wr[i / kLoadsPlane].load(stage + (i * kWaves + wave) * 1024,
                               (at + 16 * piece >= stop ? kOutside : off_n) + i % kLoadsPlane * step_n, at);
    else
      held[i] = fetch(wb[i / kLoadsPlane] + least(row_n(i), rows_n - 1) * p.w_stride, at);
  };
  const auto load_m = [&](char* stage, int c, int i) {
    const int at = c * kLinearChunk;
    if constexpr (ALIGNED)
      xr.load(stage + (i * kWaves + wave) * 1024, (at + 16 * piece >= stop ? kOutside : off_m) + i * step_m, at);
    else
      held[kLoadsN + i] = fetch(xb + least(row_m(i), rows_m - 1) * p.x_stride, at);
  };
  const auto start_n = [&](char* stage, int c) {
#pragma unroll
    for (int i = 0; i < kLoadsN; ++i) load_n(stage, c, i);
  };
  const auto start_m = [&](char* stage, int c) {
#pragma unroll
    for (int i = 0; i < kLoadsM; ++i) load_m(stage, c, i);
  };
  const auto put = [&](char* to_n, char* to_m) {
    if constexpr (!ALIGNED) {
#pragma unroll
      for (int i = 0; i < kLoadsN; ++i) *reinterpret_cast<u32x4*>(to_n + (i * kWaves + wave) * 1024 + lane * 16) = held[i];
#pragma unroll
      for (int i = 0; i < kLoadsM; ++i)
        *reinterpret_cast<u32x4*>(to_m + (i * kWaves + wave) * 1024 + lane * 16) = held[kLoadsN + i];
    }
  };

  const int wm = wave % WM, wn = wave / WM, row = lane & 15, group = lane >> 4;
  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  struct Operands {
    u32x4 v[TN + TM];
  } lo, hi;
  // This lane's place in the first step's operands; the second's is 64 bytes
  // on, before the permutation. It is made anew for each step (the compiler
  // would keep one in registers for every stage and step, and spill them).
  const int from = row * kLinearChunk + (group ^ (row & 7)) * 16;
  const auto operands_at = [&](int step) {
    int at = from;
    asm volatile("" : "+v"(at));
    return at ^ (64 * step);
  };
  // Operand t of a step, `at` its place: tiles of weights, then of x.
  const auto read = [&](const char* from_n, const char* from_m, int at, Operands& o, int t) {
    if (t >= TN) {
      o.v[t] = *reinterpret_cast<const u32x4*>(from_m + at + (wm * TM + t - TN) * 16 * kLinearChunk);
    } else {
      const int r = GATED ? (t >= TN / 2 ? kCols : 0) + wn * (TN / 2 * 16) + t % (TN / 2) * 16 : (wn * TN + t) * 16;
      o.v[t] = *reinterpret_cast<const u32x4*>(from_n + at + r * kLinearChunk);
    }
  };
  // A step's products, with other(0) .. other(others - 1) between the first of them.
  constexpr int kProducts = TN * TM, kRate = (TN + TM + kLoads + kProducts - 1) / kProducts;
  const auto multiply = [&](const Operands& o, int others, auto other) {
#pragma unroll
    for (int q = 0; q < kProducts; ++q) {
      acc[q / TM][q % TM] = mma<E>(o.v[q / TM], o.v[TN + q % TM], acc[q / TM][q % TM]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = q * kRate; t < (q + 1) * kRate && t < others; ++t) other(t);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Each chunk is two steps. The first step's operands of a chunk are read
  // while the second of the chunk before it is multiplied; the one barrier per
  // chunk lies between: all waves have read the chunk, whose stages take the
  // loads of x's chunk SM and the weights' chunk SN further on, and the next
  // chunk's loads have landed, of which the weights' may have had a chunk
  // longer. What is loaded and read stands between the products one by one
  // (all at the start of a step, the loads' issue held the products up: 8192 x
  // 14336 x 3584 722 -> 697 us). Chunks behind the end load nothing.
  constexpr int kLate = SN > SM ? kLoadsN : 0;  // loads of the weights that may still be under way
  if constexpr (ALIGNED) {
    each<SN>([&](auto j) {
      constexpr int k = decltype(j)::value;
      if constexpr (k < SM) start_m(stage_m(j), first + k);
      start_n(stage_n(j), first + k);
    });
    landed<kLoads*(SM - 1) + kLate>();
    barrier();
  } else {
    start_n(n_0, first);
    start_m(m_0, first);
    put(n_0, m_0);
    __syncthreads();
    start_n(n_1, first + 1);
    start_m(m_1, first + 1);
  }
#pragma unroll
  for (int t = 0; t < TN + TM; ++t) read(n_0, m_0, from, lo, t);
  int c = first;
  const auto chunk = [&](auto j) {
    constexpr int k = decltype(j)::value;
    constexpr std::integral_constant<int, k + 1> next{};
    __builtin_amdgcn_sched_barrier(0);
    const int at_hi = operands_at(1);
    multiply(lo, TN + TM, [&](int t) { read(stage_n(j), stage_m(j), at_hi, hi, t); });
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ALIGNED) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the second step's operands
      landed<kLoads*(SM - 2) + kLate>();
      barrier();
    } else {
      put(stage_n(next), stage_m(next));
      __syncthreads();
    }
    const int at_lo = operands_at(0);
    multiply(hi, TN + TM + kLoads, [&](int t) {
      if (t < kLoadsM)
        load_m(stage_m(j), c + SM, t);
      else if (t < kLoads)
        load_n(stage_n(j), c + SN, t - kLoadsM);
      else
        read(stage_n(next), stage_m(next), at_lo, lo, t - kLoads);
    });
    return ++c < end;
  };
  // Rounds of as many chunks as both operands' stages come round in, without a
  // branch between them (at a loop's head that others lead to, the compiler
  // waits for all loads), and the last ones. But for the largest tile, a round
  // of six, whose registers do not suffice for the code twice (1% there; 320 x
  // 14336 x 3584 with 128 x 256: 55 -> 50 us).
  constexpr int kRound = SM == SN ? SN : SM * SN;
  if constexpr (SM == SN) {
    while (c + kRound <= end) each<kRound>(chunk);
    if (c < end) all<kRound - 1>(chunk);
  } else {
    while (all<kRound>(chunk)) {
    }
  }

  // The sums go through LDS, two tiles of rows at a time, so that what is
  // written is whole runs of columns: a lane has the same four columns in
  // every row. The activation, a long one, stands in a loop; what waits for
  // memory does not.
  constexpr int kWidth = TN * 4, kQuads = GATED ? kWidth / 2 : kWidth;  // four columns each
  constexpr int kPart = 32 * kWidth * 16, kInN = kBytesN / kPart, kInM = kBytesM / kPart;  // a wave's bytes, waves to a stage
  static_assert(kWaves <= 2 * (kInN + kInM) && (kWidth & (kWidth - 1)) == 0, "the waves' parts of two stages");
  char* const part = wave < kInN       ? n_0 + wave * kPart
                     : wave < 2 * kInN ? n_1 + (wave - kInN) * kPart
                     : wave < 2 * kInN + kInM ? m_0 + (wave - 2 * kInN) * kPart : m_1 + (wave - 2 * kInN - kInM) * kPart;
  f32x4* const tile = reinterpret_cast<f32x4*>(part);
  const auto place = [&](int r, int q) { return tile + r * kWidth + (q ^ (r & (kWidth - 1))); };  // (spread over the banks)
  constexpr int kStride = 64 / kQuads, kRows = 32 / kStride;  // rows apart, and rows, of a lane
  const int q = lane % kQuads, r0 = lane / kQuads, n = n0 + (wn * kQuads + q) * 4;
  const bool whole = p.splits == 1, heavy = whole && (GATED || p.act != kActNone);
  const int first_row = m0 + wm * TM * 16 + r0;
  Four ahead[kRows], stored[kPlanes][1];
  const auto look_ahead = [&](int j) {
    load_residual(p, ahead, [&](int i) { return first_row + j * 16 + i * kStride; }, [&](int) { return n; });
  };
  landed();
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) load_bias(p, i, stored[i], [&](int) { return n; });
  if (whole) look_ahead(0);
  barrier();  // (the stages are free; from here on each wave keeps to its own part)
  const f32x4 bias = bias_type(p).value(stored[0][0]), up_bias = bias_type(p).value(stored[kPlanes - 1][0]);
#pragma unroll
  for (int j = 0; j < TM; j += 2) {
    const int m = first_row + j * 16;
    Four residual[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) residual[i] = ahead[i];
    if (whole && j + 2 < TM) look_ahead(j + 2);
    wave_sync();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < TN; ++i) *place(16 * h + row, 4 * i + group) = acc[i][j + h];
    wave_sync();
    if (heavy) {
#pragma nounroll
      for (int i = 0; i < kRows; ++i) {
        f32x4* at = place(r0 + i * kStride, q);
        *at = activated<GATED>(p, bias, up_bias, *at, *place(r0 + i * kStride, q + (GATED ? kQuads : 0)));
      }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (m + i * kStride >= p.rows || n >= p.n) continue;
      f32x4 y = *place(r0 + i * kStride, q);
      if (!whole) {
        store_parts<GATED>(p, split, m + i * kStride, n, y, *place(r0 + i * kStride, q + (GATED ? kQuads : 0)));
        continue;
      }
      if (!heavy) y += bias;
      store_out(p, m + i * kStride, n, y + residual_type(p).value(residual[i]));
    }
  }
}

// The splits' sums, added in their order, and finished. Bound by memory and
// the round trip: six parts of 320 x 3584 in 6.6 us, 28 MB that the caches hold
// in part.
constexpr int kJoinThreads = 256;

template <bool GATED>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(LinearParams p) {
  constexpr int kPlanes = GATED ? 2 : 1;
  const int quads = (p.n + 3) / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kJoinThreads + threadIdx.x;
  if (i >= static_cast<int64_t>(quads) * p.rows) return;
  const int m = static_cast<int>(i / quads), n = static_cast<int>(i % quads) * 4;
  Four bias[kPlanes][1], residual[1];
#pragma unroll
  for (int q = 0; q < kPlanes; ++q) load_bias(p, q, bias[q], [&](int) { return n; });
  load_residual(p, residual, [&](int) { return m; }, [&](int) { return n; });
  f32x4 y[kPlanes];
#pragma unroll
  for (int q = 0; q < kPlanes; ++q) {
    y[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t step = part_at(p, 1, q, kPlanes, m, n) - part_at(p, 0, q, kPlanes, m, n);
    const float* from = p.part + part_at(p, 0, q, kPlanes, m, n);
    int s = 0;
    if (p.n % 4 == 0)
      for (; s + 4 <= p.splits; s += 4, from += 4 * step) {
        f32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const f32x4u*>(from + i * step);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[q] += v[i];
      }
    for (; s < p.splits; ++s, from += step) y[q] += load_row4(from, 0, columns(p, n), false);
  }
  store_out(p, m, n, activated<GATED>(p, bias_type(p).value(bias[0][0]), bias_type(p).value(bias[kPlanes - 1][0]), y[0],
                                      y[kPlanes - 1]) + residual_type(p).value(residual[0]));
}

// ---- norm --------------------------------------------------------------------

constexpr int kRmsThreads = 256;
template <typename E>
__device__ __forceinline__ void store_row8(E* dst, int count, const float (&x)[8]) {
  if (count == 8) {
    if constexpr (sizeof(E) == 2) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      *reinterpret_cast<u32x4u*>(dst) = w;
    } else {
      *reinterpret_cast<f32x4u*>(dst) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4u*>(dst + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < count) dst[i] = static_cast<E>(x[i]);
}

// Eight elements as they are stored.
template <typename E>
struct Piece {
  u32x4 v[sizeof(E) / 2];

  __device__ __forceinline__ void load(const E* src, int count) {  // (at most 8; the others are zero)
    if (count == 8) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(E) / 2); ++i) v[i] = reinterpret_cast<const u32x4u*>(src)[i];
      return;
    }
    E e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < count ? src[i] : static_cast<E>(0.f);
    __builtin_memcpy(v, e, sizeof(v));
  }
  __device__ __forceinline__ void ones() {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(E) / 2); ++i) v[i] = u32x4(sizeof(E) == 2 ? 0x3F803F80u : 0x3F800000u);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(E) == 2) {
      return __builtin_bit_cast(float, i % 2 ? v[0][i / 2] & 0xFFFF0000u : v[0][i / 2] << 16);
    } else {
      const uint32_t bits = v[i / 4][i % 4];  // (a copy: the cast of an element itself takes the first)
      return __builtin_bit_cast(float, bits);
    }
  }
  template <typename T>
  __device__ __forceinline__ T squares() const {
    T s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += static_cast<T>(at(i)) * static_cast<T>(at(i));
    return s;
  }
};

template <typename T, typename E, typename O>
__device__ __forceinline__ void rms_store(O* dst, int count, const Piece<E>& x, const Piece<E>& w, T scale) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = static_cast<float>(static_cast<T>(x.at(i)) * scale * static_cast<T>(w.at(i)));
  store_row8(dst, count, y);
}

__device__ __forceinline__ float rms_scale(const RmsParams& p, float sum) {
  return 1.f / sqrtf(sum / static_cast<float>(p.len) + p.eps);
}
__device__ __forceinline__ double rms_scale(const RmsParams& p, double sum) {
  return 1.0 / sqrt(sum / static_cast<double>(p.len) + static_cast<double>(p.eps));
}

// out[i] = x[i] / sqrt(mean of x^2 + eps) * weight[i]. Rows of whole pieces of
// 8, at most P to a lane: a wave to a row, which stays in registers as it is
// stored, with no barrier, and the weights for all of the wave's rows. Bound by
// memory (16384 rows of 3584 in bf16 46 us, a copy of as many bytes 47; with a
// workgroup to a row, 55), for few rows by the launch.
//
// T, in which squares, sum, scale and products are: float where eps is at
// least kRmsLeastEps. What squares lose below 2^-149 is then at most 2^-30 of
// mean + eps. A smaller eps may leave the scale to a row whose squares vanish in
// fp32, or whose scale passes its range: double (16384 rows of 3584 in bf16 56
// us, in float 46; of 2048 27 and 25).
constexpr float kRmsLeastEps = 0x1p-120f;
constexpr int kRmsRows = kRmsThreads / 64;  // to a workgroup at a time

template <typename T, typename E, typename O, int P>
__global__ __launch_bounds__(kRmsThreads) void rms_wave_kernel(RmsParams p) {
  const int pieces = p.len / 8, lane = static_cast<int>(threadIdx.x) % 64;
  const E* weight = static_cast<const E*>(p.weight);
  // (Lanes behind the row's end load its last piece, and neither add nor store it.)
  const auto at = [&](int i) { return 8 * least(lane + 64 * i, pieces - 1); };
  Piece<E> w[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    w[i].ones();
    if (weight && 64 * i < pieces) w[i].load(weight + at(i), 8);
  }
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRmsRows + wave_id(); row < p.rows;
       row += static_cast<int64_t>(gridDim.x) * kRmsRows) {
    const E* x = static_cast<const E*>(p.x) + row * p.x_stride;
    O* out = static_cast<O*>(p.out) + row * p.out_stride;
    Piece<E> held[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (64 * i < pieces) held[i].load(x + at(i), 8);
    T sum = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (64 * i >= pieces) continue;
      const T s = held[i].template squares<T>();
      sum += lane + 64 * i < pieces ? s : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    const T scale = rms_scale(p, sum);
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (lane + 64 * i < pieces) rms_store(out + 8 * (lane + 64 * i), 8, held[i], w[i], scale);
  }
}

// Other rows (and those of over 4096: 4096 rows of 6144 in 20.9 us, a wave to
// each 25.4): a workgroup to each, which is read twice.
template <typename T, typename E, typename O>
__global__ __launch_bounds__(kRmsThreads) void rms_long_kernel(RmsParams p) {
  __shared__ T red[2][kRmsThreads / 64];
  const int pieces = (p.len - 1) / 8 + 1, tid = static_cast<int>(threadIdx.x);
  const auto count = [&](int at) { return at + 1 < pieces ? 8 : p.len - 8 * at; };
  const E* weight = static_cast<const E*>(p.weight);
  int turn = 0;  // (the sums' place alternates: one barrier per row)
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
    const E* x = static_cast<const E*>(p.x) + row * p.x_stride;
    O* out = static_cast<O*>(p.out) + row * p.out_stride;
    T sum = 0;
    Piece<E> piece, w;
    w.ones();
    for (int at = tid; at < pieces; at += kRmsThreads) {
      piece.load(x + 8 * at, count(at));
      sum += piece.template squares<T>();
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63) == 0) red[turn][tid / 64] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int i = 0; i < kRmsThreads / 64; ++i) sum += red[turn][i];
    const T scale = rms_scale(p, sum);
    for (int at = tid; at < pieces; at += kRmsThreads) {
      piece.load(x + 8 * at, count(at));
      if (weight) w.load(weight + 8 * at, count(at));
      rms_store(out + 8 * at, count(at), piece, w, scale);
    }
  }
}

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

}  // namespace

template <typename E, bool GATED, bool ALIGNED>
static hipError_t launch_thin(const LinearParams& p, const LinearPlan& plan, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.m_tiles * p.n_tiles * p.splits));
#define TTS_THIN(BM, BN)                                                                                            \
  if (plan.bm == BM && plan.bn == BN) {                                                                             \
    hipLaunchKernelGGL((thin_kernel<E, BM, BN, ALIGNED ? thin_stages(BM, BN) : 2, GATED, ALIGNED>), grid,          \
                       dim3(kThinThreads), 0, stream, p);                                                            \
    return hipGetLastError();                                                                                        \
  }
  if constexpr (!GATED) {
    TTS_THIN(16, 16)
    TTS_THIN(32, 16)
    TTS_THIN(16, 48)
    TTS_THIN(32, 48)
  }
  TTS_THIN(16, 32)
  TTS_THIN(32, 32)
  TTS_THIN(64, 32)
  TTS_THIN(16, 64)
  TTS_THIN(32, 64)
  TTS_THIN(64, 64)
#undef TTS_THIN
  return hipErrorInvalidValue;
}

// (A plan whose tile has no kernel is refused: a grid counted in other tiles
// than the kernel's would leave the operands.)
template <typename E, bool GATED, bool ALIGNED>
static hipError_t launch_tiles(const LinearParams& p, const LinearPlan& plan, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.m_tiles * p.n_tiles * p.splits));
#define TTS_TILE(BM, BN, WM, WN, SM, SN)                                                                                  \
  if (plan.bm == BM && plan.bn == BN && plan.tile == 10 * SM + SN && plan.threads == 64 * WM * WN) {                       \
    hipLaunchKernelGGL((tile_kernel<E, BM, BN, WM, WN, SM, SN, GATED, ALIGNED>), grid, dim3(64 * WM * WN), 0, stream, p); \
    return hipGetLastError();                                                                                              \
  }
  if constexpr (ALIGNED && sizeof(E) == 2) {
    TTS_TILE(256, 256, 2, 4, 2, 3)
    TTS_TILE(128, 256, 2, 4, 3, 3)
    TTS_TILE(128, 128, 2, 2, 4, 4)
    TTS_TILE(64, 128, 1, 4, 3, 3)
  } else {
    TTS_TILE(128, 128, 2, 2, 2, 2)
  }
#undef TTS_TILE
  return hipErrorInvalidValue;
}

template <typename E, bool GATED>
static hipError_t launch_linear_t(LinearParams p, const LinearPlan& plan, bool aligned, hipStream_t stream) {
  p.splits = plan.splits;
  p.chunks = plan.chunks;
  p.m_tiles = ceil_div(p.rows, plan.bm);
  p.n_tiles = ceil_div(static_cast<int64_t>(p.n) * (GATED ? 2 : 1), plan.bn);
  hipError_t e;
  if (plan.tile == 0)
    e = aligned ? launch_thin<E, GATED, true>(p, plan, stream) : launch_thin<E, GATED, false>(p, plan, stream);
  else
    e = aligned ? launch_tiles<E, GATED, true>(p, plan, stream) : launch_tiles<E, GATED, false>(p, plan, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t items = static_cast<int64_t>((p.n + 3) / 4) * p.rows;
  hipLaunchKernelGGL(join_kernel<GATED>, dim3(static_cast<unsigned>((items + kJoinThreads - 1) / kJoinThreads)),
                     dim3(kJoinThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearParams& p, const LinearPlan& plan, bool gated, bool aligned, hipStream_t stream) {
  if (p.in_bf16)
    return gated ? launch_linear_t<uint16_t, true>(p, plan, aligned, stream)
                 : launch_linear_t<uint16_t, false>(p, plan, aligned, stream);
  return gated ? launch_linear_t<float, true>(p, plan, aligned, stream)
               : launch_linear_t<float, false>(p, plan, aligned, stream);
}

template <typename T, typename E, typename O>
static hipError_t launch_rms_t(const RmsParams& p, hipStream_t stream) {
  const dim3 block(kRmsThreads);
  // As many workgroups as run at once take the rows in turn.
  const int64_t groups = (static_cast<int64_t>(p.rows) + kRmsRows - 1) / kRmsRows;
  const int lane_pieces = p.len % 8 == 0 ? ceil_div(p.len, 512) : 0;  // 0: rows that do not end with a piece
  constexpr int kMost = 256 * 8;
  const dim3 grid(static_cast<unsigned>(groups < kMost ? groups : kMost));
  if (lane_pieces == 0 || lane_pieces > 8)
    hipLaunchKernelGGL((rms_long_kernel<T, E, O>), dim3(static_cast<unsigned>(p.rows < kMost ? p.rows : kMost)), block, 0,
                       stream, p);
  else if (lane_pieces <= 2)
    hipLaunchKernelGGL((rms_wave_kernel<T, E, O, 2>), grid, block, 0, stream, p);
  else if (lane_pieces <= 4)
    hipLaunchKernelGGL((rms_wave_kernel<T, E, O, 4>), grid, block, 0, stream, p);
  else if (lane_pieces <= 6)
    hipLaunchKernelGGL((rms_wave_kernel<T, E, O, 6>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((rms_wave_kernel<T, E, O, 8>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_rms_of(const RmsParams& p, hipStream_t stream) {
  if (p.in_bf16) return p.out_bf16 ? launch_rms_t<T, __bf16, __bf16>(p, stream) : launch_rms_t<T, __bf16, float>(p, stream);
  return p.out_bf16 ? launch_rms_t<T, float, __bf16>(p, stream) : launch_rms_t<T, float, float>(p, stream);
}

hipError_t launch_rms(const RmsParams& p, hipStream_t stream) {
  return p.eps >= kRmsLeastEps ? launch_rms_of<float>(p, stream) : launch_rms_of<double>(p, stream);
}

}  // namespace tts
