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

// How a product is launched: `tile` 0: small tiles, whose workgroup deals the
// inner dimension to its waves; else large tiles, of so many stages.
struct LinearPlan {
  int tile;
  int bm, bn;  // rows of x and rows of weights to a workgroup
  int splits, chunks;
  int64_t groups;  // workgroups of one split
  size_t workspace;
};

constexpr int kLinearChunk = 128;  // bytes of a row to a step of the large tiles
constexpr int kThinChunk = 256;    // and of the small ones

// `aligned`: every row of both operands starts at a multiple of 16 bytes.
LinearPlan linear_plan(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated, bool aligned);

// The most that a call of up to `rows` rows needs.
size_t linear_workspace(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated);

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
