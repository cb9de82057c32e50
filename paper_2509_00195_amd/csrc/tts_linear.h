// Parameters and launch plan of the projections. Plain C++, shared with the C
// ABI's host code.
#pragma once

#include <cstddef>
#include <cstdint>

namespace tts {

enum LinearAct : int { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3, kActGeluTanh = 4 };

struct LinearParams {
  const void* x;
  const void* w[2];     // gated: gate, up; else the weights and null
  const void* bias[2];  // null: none
  const void* residual;
  void* out;
  float* part;                                // partial sums [split][gate, up][row][column], when split
  int64_t x_stride, w_stride;                 // bytes between rows
  int64_t residual_stride, out_stride;        // elements between rows
  int32_t rows, n;
  int32_t k_bytes;                            // of one row of x or of the weights
  int32_t act;
  int32_t in_bf16, out_bf16;
  int32_t splits, chunks;                     // parts of the inner dimension, chunks to a part
  int32_t m_tiles, n_tiles;
};

// How a product is launched. tile 0: small tiles, whose workgroup deals the
// inner dimension to its waves; else large tiles, x's and the weights' stages
// as two digits.
struct LinearPlan {
  int tile;
  int bm, bn;  // rows of x and rows of weights to a workgroup
  int splits, chunks;
  int64_t groups;  // workgroups of one split
  int threads;     // of a workgroup
  size_t workspace;

  bool fits() const { return groups * threads < int64_t{1} << 32; }  // (one launch's threads; split calls are smaller)
};

constexpr int kLinearChunk = 128;  // bytes of a row to a step of the large tiles
constexpr int kThinChunk = 256;    // and of the small ones
constexpr int kThinThreads = 256;  // of whose workgroups

// The small tiles that there are. (64 x 48 has no third stage, and was slower
// than 64 x 32 at every size; 64 x 16 was nowhere the best.)
constexpr bool thin_has(int bm, int bn, bool gated) {
  return gated ? bn == 32 || bn == 64 : bn == 32 || bn == 64 || bm < 64;
}

// Their stages: as many as leave room for two workgroups on a compute unit
// (160 KB of LDS), at most eight.
constexpr int thin_stages(int bm, int bn) {
  const int n = 78 * 1024 / ((bm + bn) * kThinChunk);
  return n > 8 ? 8 : n;
}

// `aligned`: every row of both operands starts at a multiple of 16 bytes.
LinearPlan linear_plan(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated, bool aligned);

// What a call of up to `rows` rows needs at most.
size_t linear_workspace(int32_t rows, int32_t n, int32_t k_bytes, bool gated);

struct RmsParams {
  const void* x;
  const void* weight;  // null: ones
  void* out;
  int64_t x_stride, out_stride;  // elements
  int32_t rows, len;
  int32_t in_bf16, out_bf16;
  float eps;
};

}  // namespace tts
