// Parameters of the rotating append. Plain C++, shared with the C ABI's host
// code.
#pragma once

#include <cstdint>

namespace tts {

constexpr int kRopeTile = 4096;   // elements (tokens x heads x head dims) of a K or V part
constexpr int kRopeTasks = 1024;  // units of the query rows to a part

struct RopeParams {
  const void* q;  // null: no queries
  const void* k_new;
  const void* v_new;
  void* q_out;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  const int32_t* tok_offsets;            // null: one token per sequence
  const int32_t* positions;              // null: the token's index in its sequence
  const int32_t* block_tables;
  const int32_t* seq_lens;
  const float* cos;
  const float* sin;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  int64_t item0;  // set by the launch, as is what follows max_pos
  int32_t num_seqs;
  int32_t num_tokens;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t hq;
  int32_t hkv;
  int32_t head_dim;
  int32_t rot;  // 0: no rotation
  int32_t interleaved;
  int32_t max_pos;
  int32_t heads_per, kv_parts;
  int32_t q_wide, k_wide, v_wide;
};

}  // namespace tts
