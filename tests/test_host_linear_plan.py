"""The launch plan of the projections, compiled by itself under AddressSanitizer and UndefinedBehaviorSanitizer (CPU)."""

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_00195_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "tts_linear.h"
using namespace tts;

#define CHECK(x) do { if (!(x)) { std::printf("%s: rows %d n %d k_bytes %d f32 %d gated %d aligned %d: tile %d %d x %d " \
  "splits %d chunks %d\n", #x, rows, n, k_bytes, f32, gated, aligned, p.tile, p.bm, p.bn, p.splits, p.chunks); std::exit(1); } } while (0)

static void check(int rows, int n, int k_bytes, bool f32, bool gated, bool aligned, int most_rows) {
  const LinearPlan p = linear_plan(rows, n, k_bytes, f32, gated, aligned);
  const int64_t cols = static_cast<int64_t>(n) * (gated ? 2 : 1), chunk = p.tile ? kLinearChunk : kThinChunk;
  const int64_t total = (k_bytes + chunk - 1) / chunk;
  // a kernel of these tiles
  if (p.tile == 0) CHECK((p.bm == 16 || p.bm == 32 || p.bm == 64) && p.bn % 16 == 0 && p.bn <= 64 && thin_has(p.bm, p.bn, gated));
  else if (f32 || !aligned) CHECK(p.tile == 22 && p.bm == 128 && p.bn == 128);
  else CHECK((p.tile == 23 && p.bm == 256 && p.bn == 256) ||
             (p.tile == 33 && p.bm == 128 && p.bn == 256) || (p.tile == 44 && p.bm == 128 && p.bn == 128) ||
             (p.tile == 33 && p.bm == 64 && p.bn == 128));
  // every part has chunks, and together they have all
  CHECK(p.splits >= 1 && p.chunks >= 1 && static_cast<int64_t>(p.splits) * p.chunks >= total);
  CHECK(static_cast<int64_t>(p.splits - 1) * p.chunks < total);
  CHECK(p.groups == ((rows + static_cast<int64_t>(p.bm) - 1) / p.bm) * ((cols + p.bn - 1) / p.bn));
  CHECK(p.workspace == (p.splits == 1 ? 0 : static_cast<size_t>(p.splits) * rows * cols * 4));
  CHECK(p.workspace <= linear_workspace(rows, n, k_bytes, gated));
  if (most_rows >= rows) CHECK(p.workspace <= linear_workspace(most_rows, n, k_bytes, gated));
  CHECK(linear_workspace(rows, n, k_bytes, gated) <= linear_workspace(rows < (1 << 30) ? 2 * rows : rows, n, k_bytes, gated));
}

int main() {
  std::mt19937 gen(7);
  const auto log = [&](double a, double b) {
    return static_cast<int>(std::exp(std::uniform_real_distribution<double>(std::log(a), std::log(b))(gen)));
  };
  for (int i = 0; i < 20000; ++i) {
    const bool f32 = gen() % 2, gated = gen() % 2, aligned = gen() % 2;
    const int rows = log(1, 20000), n = log(1, 40000), k_bytes = (f32 ? 4 : 2) * log(1, 30000);
    check(rows, n, k_bytes, f32, gated, aligned, rows + log(1, 5000));
  }
  for (int rows : {1, 17, 2147483647})
    for (int n : {1, 1 << 26})
      for (int k_bytes : {2, 4, 1 << 30})
        for (int v = 0; v < 8; ++v)
          if (k_bytes % (v & 1 ? 4 : 2) == 0) check(rows, n, k_bytes, v & 1, v & 2, v & 4, 2147483647);
  std::printf("ok\n");
}
"""


def test_plans_and_workspaces(tmp_path):
    from paper_2509_00195_amd.build import SANITIZE

    src, exe = tmp_path / "main.cpp", tmp_path / "plan"
    src.write_text("#include <cmath>\n" + MAIN)
    subprocess.run([os.environ.get("CXX_HOST", "g++"), "-std=c++17", *SANITIZE, f"-I{CSRC}", str(src),
                    os.path.join(CSRC, "tts_linear.cpp"), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout[-1500:] + r.stderr[-1500:]
