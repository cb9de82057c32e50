// Parameters of the ragged prefill attention. Plain C++, shared with the C
// ABI's host code.
#pragma once

#include <cstddef>
#include <cstdint>

namespace tts {

// Query rows of a workgroup: rows of one sequence and one KV head, token by
// token with the head's query heads side by side.
constexpr int kPrefillRows = 128;
// Splits of a tile of rows over the tokens, at most.
constexpr int kPrefillMaxSplit = 32;

struct PrefillParams {
  const void* q;
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  const int32_t* tok_offsets;
  const int32_t* block_tables;
  const int32_t* seq_lens;
  void* out;
  float* part_o;   // [nsplit][num_tokens * hq][D]: o (not normalised)
  float* part_ml;  // [nsplit][num_tokens * hq][2]: reference (log2 units), sum
  int64_t unit0;   // set by the launch
  int64_t units;   // items x KV heads x splits
  int32_t num_seqs;
  int32_t num_tokens;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t max_seq_len;
  int32_t hq;
  int32_t hkv;
  int32_t g;
  int32_t nsplit;
  int32_t out_bf16;
  float scale_log2;
};

// Items (tiles of rows, some empty) of a call: sequence b has items
// [off[b] * g / kPrefillRows + b, the same of b + 1).
inline int64_t prefill_items(int64_t num_seqs, int64_t num_tokens, int64_t g) {
  return num_tokens * g / kPrefillRows + num_seqs;
}

}  // namespace tts
