// Cache geometry, types and conversions shared by the HIP kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tts {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kTok = 16;      // tokens per KV block
constexpr int kMxGroup = 32;  // head dims under one scale of a 4-bit cache

enum KvKind : int { kKvF32 = 0, kKvBf16 = 1, kKvFp8 = 2, kKvMx4 = 3 };

// One (block, head) of K or V: K token-major, V dim-major. 4-bit caches:
// two elements to a byte, lower half first, and behind the block's codes one
// scale byte per 32 dims of a token (K [16][D / 32], V [D / 32][16]).
template <int D, int KV>
struct KvGeo {
  static constexpr int bits = KV == kKvF32 ? 32 : (KV == kKvBf16 ? 16 : (KV == kKvFp8 ? 8 : 4));
  static constexpr int row_bytes = D * bits / 8;       // one token of K
  static constexpr int code_bytes = kTok * row_bytes;  // the elements
  static constexpr int blk_bytes = code_bytes + (KV == kKvMx4 ? kTok * D / kMxGroup : 0);
  static constexpr int vrow_bytes = kTok * bits / 8;   // one dim of V (16 tokens)
  static constexpr int vhalf_bytes = vrow_bytes / 2;   // eight tokens of it
};

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));  // RNE
}

// x + both halves, two fp32 roundings at most (one instruction, against an
// add for each and their unpacking).
__device__ __forceinline__ float add_bf16x2(uint32_t pair, float x) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), x,
                                         false);
}

__device__ __forceinline__ float bf16_to_f32(uint16_t b) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(b) << 16);
}

// Two OCP E4M3 codes (byte pair kHi of w) -> two bf16 in one dword, in one
// conversion instruction with unit scale. Every E4M3 value fits bf16
// exactly, so the conversion is exact.
template <bool kHi>
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHi));
}

__device__ __forceinline__ uint4 fp8x8_to_bf16x8(uint2 w) {
  return uint4{fp8x2_to_bf16x2<false>(w.x), fp8x2_to_bf16x2<true>(w.x), fp8x2_to_bf16x2<false>(w.y),
               fp8x2_to_bf16x2<true>(w.y)};
}

// Byte kByte of w, an E8M0 scale 2^(byte - 127), as the scale operand of the
// conversions from E2M1, which read its exponent bits (255: NaN, and so are
// the converted values; 0: 2^-127).
template <int kByte>
__device__ __forceinline__ float mx_scale(uint32_t w) {
  return __builtin_bit_cast(float, ((w >> (8 * kByte)) & 0xFFu) << 23);
}

// The two E2M1 codes in byte kByte of w (lower half first) times the scale,
// as two bf16 in one dword: exact (two significant bits).
template <int kByte>
__device__ __forceinline__ uint32_t mx4x2_to_bf16x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, kByte));
}

// Eight codes under one scale (dims of a token).
__device__ __forceinline__ uint4 mx4x8_to_bf16x8(uint32_t w, float scale) {
  return uint4{mx4x2_to_bf16x2<0>(w, scale), mx4x2_to_bf16x2<1>(w, scale), mx4x2_to_bf16x2<2>(w, scale),
               mx4x2_to_bf16x2<3>(w, scale)};
}

// Eight codes each under its own scale (tokens of a dim): every pair is
// converted under either scale and a half of each result kept.
__device__ __forceinline__ uint4 mx4x8_to_bf16x8(uint32_t w, uint2 s) {
  auto mix = [](uint32_t lo, uint32_t hi) { return (lo & 0xFFFFu) | (hi & 0xFFFF0000u); };
  return uint4{mix(mx4x2_to_bf16x2<0>(w, mx_scale<0>(s.x)), mx4x2_to_bf16x2<0>(w, mx_scale<1>(s.x))),
               mix(mx4x2_to_bf16x2<1>(w, mx_scale<2>(s.x)), mx4x2_to_bf16x2<1>(w, mx_scale<3>(s.x))),
               mix(mx4x2_to_bf16x2<2>(w, mx_scale<0>(s.y)), mx4x2_to_bf16x2<2>(w, mx_scale<1>(s.y))),
               mix(mx4x2_to_bf16x2<3>(w, mx_scale<2>(s.y)), mx4x2_to_bf16x2<3>(w, mx_scale<3>(s.y)))};
}

// A value at a uniform address that the kernel does not write.
template <typename T>
__device__ __forceinline__ T scalar(const T* at) {
  typedef const T __attribute__((address_space(4))) * P;
  return *(P)(reinterpret_cast<uintptr_t>(at));
}

// The sequence whose range of items holds `item`, when sequence b's begins at
// first(b), increasing with b. Every wave looks for itself, 64 sequences at a
// step; in bounds and finite whatever the offsets hold.
template <typename F>
__device__ __forceinline__ int find_seq(int num_seqs, int64_t item, F first) {
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, hi = num_seqs;
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool le = lane == 0 || (at < hi && first(at) <= item);
    lo += (__builtin_popcountll(__builtin_amdgcn_ballot_w64(le)) - 1) * step;
    hi = hi < lo + step ? hi : lo + step;
  }
  return __builtin_amdgcn_readfirstlane(static_cast<int>(lo));
}

// Four elements of an output row from element `at` on.
__device__ __forceinline__ void store_out4(void* out, bool bf16, int64_t at, f32x4 x) {
  if (bf16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = uint2{pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w)};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = x;
}

}  // namespace tts
