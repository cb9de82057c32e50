// Launch plan of the projections: which kernel, which tiles, how many parts of
// the inner dimension. Every combination that has a kernel is priced by a
// model of the call's time, in microseconds, and the cheapest taken.
#include "tts_linear.h"

#include <cmath>

namespace tts {

namespace {

constexpr int kUnits = 256;       // compute units
constexpr int kMostSplits = 16;
constexpr int kLeastChunk = 2048;  // bytes of a row to a part, at least

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A tile that has a kernel. threads: of a workgroup. resident: workgroups that
// a compute unit holds.
// chunk: time of a chunk of the inner dimension, of one workgroup and of two
// on a compute unit, while its loads keep up (measured; a few percent of which
// the number of busy units makes).
struct Tile {
  int tile, bm, bn, threads, resident;
  double one, two;
};

// Large tiles of bf16 rows at multiples of 16 bytes: K 3584 (56 chunks) in 85 us
// at 224 of 256 units (256 x 256), 50.6 at 224 (128 x 256), 31.9 at 180 (128 x
// 128), 22.8 and 36.9 at 180 and 360 (64 x 128), less 3.5 for the launch.
constexpr Tile kTiles[] = {{23, 256, 256, 512, 1, 1.46, 0}, {33, 128, 256, 512, 1, 0.84, 0},
                           {44, 128, 128, 256, 1, 0.52, 0}, {33, 64, 128, 256, 2, 0.34, 0.60}};
// The one for other rows, fp32 by its products (4096 cycles to a chunk), rows
// that are not aligned by their way through registers.
constexpr Tile kTileF32 = {22, 128, 128, 256, 2, 1.75, 3.5}, kTileOdd = {22, 128, 128, 256, 2, 1.5, 1.5};
constexpr int kThinM[] = {16, 32, 64}, kThinN[] = {16, 32, 48, 64};

constexpr double kLaunch = 3.5, kJoin = 3.0;  // launches
constexpr double kGroup = 0.6;                // a workgroup's first loads and its epilogue
constexpr double kMemory = 5.5e6;             // bytes in a microsecond, each of the operands' once
constexpr double kCaches = 14e6;              // of the tiles, from the L2s
constexpr double kPartial = 3.2e6;            // of partial sums, written and read

struct Shape {
  int64_t rows, cols;  // (gated: both planes' columns)
  int32_t k_bytes;
  bool f32, aligned;
};

double bytes_of(const Shape& s) {
  return (static_cast<double>(s.rows) + static_cast<double>(s.cols)) * s.k_bytes;
}

// The best number of parts for a tile, and its time.
double best_splits(const Shape& s, int bm, int bn, int chunk_bytes, int resident, double one, double two, int* splits) {
  const int64_t groups = ceil_div(s.rows, bm) * ceil_div(s.cols, bn), slots = static_cast<int64_t>(kUnits) * resident;
  const int64_t total = ceil_div(s.k_bytes, chunk_bytes);
  const double once = bytes_of(s) / kMemory, drawn = static_cast<double>(groups * (bm + bn)) * s.k_bytes / kCaches;
  const double memory = once > drawn ? once : drawn;
  double best = 1e30;
  for (int n = 1; n <= kMostSplits; n = n < 4 ? n + 1 : (n < 8 ? n + 2 : n + 4)) {
    if (n > 1 && (n * groups > slots || s.k_bytes / n < kLeastChunk)) break;
    const int64_t all = n * groups, rounds = ceil_div(all, slots);
    const double chunk = resident > 1 && all > kUnits ? two : one;
    const double work = static_cast<double>(rounds) * (static_cast<double>(ceil_div(total, n)) * chunk + kGroup);
    // The longer of the two, and a little more where they are near each other.
    double t = std::sqrt(std::sqrt(work * work * work * work + memory * memory * memory * memory)) + kLaunch;
    if (n > 1) t += kJoin + static_cast<double>(n) * static_cast<double>(s.rows * s.cols) * 4 / kPartial;
    if (t < best) best = t, *splits = n;
  }
  return best;
}

// A small tile's chunk: S - 1 chunks in flight cover a round trip of 0.62 us;
// a unit draws 75 bytes in a nanosecond from its L2 for one workgroup, 96 for
// two; a step takes 0.12 us at least. Rows that are not aligned pass through
// registers, a chunk ahead: 0.1 us to each of a thread's loads, and a round
// trip to memory where the operands are more than the caches hold near by.
// fp32 products are eight times slower (0.053 us to a step's 16 x 16 tile).
void thin_chunk(const Shape& s, int bm, int bn, double* one, double* two) {
  const auto most = [](double a, double b) { return a > b ? a : b; };
  const int loads = (bm + bn) / 16, products = bm * bn / 256;
  const double stage = (bm + bn) * kThinChunk, product = (s.f32 ? 0.053 : 0.0067) * products;
  if (s.aligned) {
    *one = most(most(0.62 / (thin_stages(bm, bn) - 1), 0.12), most(stage / 75e3, product));
    *two = most(most(*one, 0.23), most(2 * stage / 96e3, 2 * product));
  } else {
    const double far = bytes_of(s) / 20e6;
    *one = most(most(0.1 * loads, 0.2 + 0.4 * (far < 1 ? far : 1)), product);
    *two = most(most(*one, 0.15 * loads), 2 * product);
  }
}

}  // namespace

LinearPlan linear_plan(int32_t rows, int32_t n, int32_t k_bytes, bool f32, bool gated, bool aligned) {
  const int planes = gated ? 2 : 1;
  const Shape s{rows, static_cast<int64_t>(n) * planes, k_bytes, f32, aligned};
  LinearPlan r{};
  double best = 0;
  // (A tile whose workgroups pass one launch is taken only where all do.)
  const auto offer = [&](const Tile& t, int chunk_bytes) {
    LinearPlan q{t.tile, t.bm, t.bn, 1, 0, ceil_div(rows, t.bm) * ceil_div(s.cols, t.bn), t.threads, 0};
    const double us = best_splits(s, t.bm, t.bn, chunk_bytes, t.resident, t.one, t.two, &q.splits);
    if (r.threads == 0 || (q.fits() != r.fits() ? q.fits() : us < best)) {
      best = us;
      r = q;
    }
  };
  if (f32 || !aligned)
    offer(f32 ? kTileF32 : kTileOdd, kLinearChunk);
  else
    for (const Tile& t : kTiles) offer(t, kLinearChunk);
  for (int bm : kThinM)
    for (int bn : kThinN) {
      if (!thin_has(bm, bn, gated) || (bm > 16 && bm >= 2 * static_cast<int64_t>(rows))) continue;
      double one, two;
      thin_chunk(s, bm, bn, &one, &two);
      offer({0, bm, bn, kThinThreads, 2, one, two}, kThinChunk);
    }
  const int64_t total = ceil_div(k_bytes, r.tile ? kLinearChunk : kThinChunk);
  r.chunks = static_cast<int>(ceil_div(total, r.splits));
  r.splits = static_cast<int>(ceil_div(total, r.chunks));
  r.workspace = r.splits == 1 ? 0 : static_cast<size_t>(r.splits) * planes * rows * n * sizeof(float);
  return r;
}

size_t linear_workspace(int32_t rows, int32_t n, int32_t k_bytes, bool gated) {
  // A bound over every plan: splits times tiles are at most the workgroups
  // that run at once, and splits at most what the inner dimension allows.
  const int64_t cols = static_cast<int64_t>(n) * (gated ? 2 : 1);
  const int64_t allowed = k_bytes / kLeastChunk < kMostSplits ? k_bytes / kLeastChunk : kMostSplits;
  if (allowed < 2) return 0;
  int64_t most = 0;  // rows of partial sums, over all splits
  const auto offer = [&](int bm, int bn, int resident) {
    const int64_t places = kUnits * resident / ceil_div(cols, bn);  // splits times tiles of rows
    if (places < 2) return;
    int64_t sums = places * bm;  // (each tile of rows at most bm of them)
    if (sums > allowed * rows) sums = allowed * rows;
    if (sums > most) most = sums;
  };
  for (const Tile& t : kTiles) offer(t.bm, t.bn, t.resident);
  offer(kTileOdd.bm, kTileOdd.bn, kTileOdd.resident);
  for (int bm : kThinM)
    for (int bn : kThinN)
      if (thin_has(bm, bn, gated)) offer(bm, bn, 2);
  return static_cast<size_t>(most) * cols * sizeof(float);
}

}  // namespace tts
