"""Products of so many rows that tiles pass one launch's 2^32 threads: a plan takes another tile where one fits (CPU)."""

import ctypes as C
import os
import subprocess

from paper_2509_00195_amd import tts as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_00195_amd", "csrc")

MAIN = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include "tts_linear.h"
using namespace tts;

int main() {
  std::mt19937 gen(11);
  const auto log = [&](double a, double b) {
    return static_cast<int>(std::exp(std::uniform_real_distribution<double>(std::log(a), std::log(b))(gen)));
  };
  int tall = 0, refused = 0;
  for (int i = 0; i < 20000; ++i) {
    const bool f32 = gen() % 2, gated = gen() % 2, aligned = gen() % 2;
    const int rows = log(1 << 20, 2147483647.0), n = log(1, 1000), k_bytes = (f32 ? 4 : 2) * log(1, 4000);
    const LinearPlan p = linear_plan(rows, n, k_bytes, f32, gated, aligned);
    const int64_t cols = static_cast<int64_t>(n) * (gated ? 2 : 1);
    const auto fits = [&](int bm, int bn, int threads) {
      return ((rows + int64_t{bm} - 1) / bm) * ((cols + bn - 1) / bn) * threads < int64_t{1} << 32;
    };
    bool any = fits(128, 128, 256), all = true;
    if (!f32 && aligned) any = any || fits(256, 256, 512) || fits(128, 256, 512) || fits(64, 128, 256);
    for (int bm : {16, 32, 64})
      for (int bn : {16, 32, 48, 64})
        if (thin_has(bm, bn, gated)) {
          any = any || fits(bm, bn, 256);
          all = all && fits(bm, bn, 256);
        }
    if (any != fits(p.bm, p.bn, p.threads) || any != p.fits()) {
      std::printf("rows %d n %d k_bytes %d f32 %d gated %d aligned %d: %d x %d of %d threads\n", rows, n, k_bytes, f32, gated,
                  aligned, p.bm, p.bn, p.threads);
      return 1;
    }
    tall += any && !all;
    refused += !any;
  }
  std::printf("%d %d ok\n", tall, refused);
  return tall > 1000 && refused > 100 ? 0 : 1;
}
"""


def test_a_tile_that_fits_is_taken(tmp_path):
    from paper_2509_00195_amd.build import SANITIZE

    src, exe = tmp_path / "main.cpp", tmp_path / "plan"
    src.write_text(MAIN)
    subprocess.run([os.environ.get("CXX_HOST", "g++"), "-std=c++17", *SANITIZE, f"-I{CSRC}", str(src),
                    os.path.join(CSRC, "tts_linear.cpp"), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout[-1500:] + r.stderr[-1500:]


def test_what_no_tile_fits_is_refused():
    a = 1 << 20
    d = T.make_linear(64, 1 << 20)
    assert T.load().tts_linear(C.byref(d), (1 << 31) - 1, a, 64, a, 64, None, None, 0, a, 1 << 20, None, 0,
                               None) == T.TTS_ERR_UNSUPPORTED
