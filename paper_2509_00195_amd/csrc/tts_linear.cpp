// Launch plan of the projections: which kernel, which tiles, how many parts
// of the inner dimension.
#include "tts_linear.h"

namespace tts {

namespace {

constexpr int kUnits = 256;  // compute units
constexpr int kLeast = 16;   // chunks to a part of the inner dimension, at least

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

}  // namespace

LinearPlan linear_plan(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated, bool aligned) {
  LinearPlan r{};
  const int planes = gated ? 2 : 1;
  const int64_t cols = static_cast<int64_t>(n) * planes;
  int slots = 2 * kUnits;  // workgroups that run at once
  if (rows <= 64) {
    r.tile = 0;
    r.bm = rows <= 16 ? 16 : (rows <= 32 ? 32 : 64);
    r.bn = cols >= 8192 ? 64 : (gated || cols >= 4096 ? 32 : 16);
  } else {
    const bool wide = aligned && !f32 && static_cast<int64_t>(ceil_div(rows, 256)) * ceil_div(cols, 256) >= kUnits;
    r.bm = r.bn = wide ? 256 : 128;
    r.tile = 2;
    if (wide) slots = kUnits;
  }
  const int total = ceil_div(k_bytes, r.tile ? kLinearChunk : kThinChunk);
  const int64_t groups = static_cast<int64_t>(ceil_div(rows, r.bm)) * ceil_div(cols, r.bn);
  int64_t splits = groups >= slots ? 1 : slots / groups;
  if (splits > total / kLeast) splits = total / kLeast;
  if (splits < 1) splits = 1;
  r.chunks = ceil_div(total, splits);
  r.splits = ceil_div(total, r.chunks);
  r.groups = groups;
  r.workspace = r.splits == 1 ? 0 : static_cast<size_t>(r.splits) * planes * rows * n * sizeof(float);
  return r;
}

size_t linear_workspace(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated) {
  // A band of 128 rows has one number of splits, so its last count needs the
  // most; from the first unsplit band on none is split.
  size_t most = 0;
  for (int64_t band = 16; ; band = band < 64 ? 2 * band : (band == 64 ? 128 : band + 128)) {
    const int32_t m = band < rows ? static_cast<int32_t>(band) : rows;
    for (int aligned = 0; aligned < 2; ++aligned) {
      const LinearPlan plan = linear_plan(m, n, k_bytes, f32, gated, aligned != 0);
      if (plan.workspace > most) most = plan.workspace;
      if (m > 64 && plan.splits == 1) return most;
    }
    if (m == rows) return most;
  }
}

}  // namespace tts
