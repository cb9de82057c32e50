"""The shapes that stand for each kernel of the projections get that kernel, and there is no other that a call gets (CPU)."""

import os
import subprocess

from tests._linear_tiles import TILES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_00195_amd", "csrc")

MAIN = r"""
#include <cmath>
#include <cstdio>
#include <random>
#include <set>
#include <tuple>
#include "tts_linear.h"
using namespace tts;

static std::tuple<int, int, int, int, int, int, int> kernel_of(int m, int k, int n, bool f32, bool gated, bool aligned) {
  const LinearPlan p = linear_plan(m, n, k * (f32 ? 4 : 2), f32, gated, aligned);
  return {f32, gated, p.tile, p.bm, p.bn, aligned, p.splits > 1};
}

static void print(const std::tuple<int, int, int, int, int, int, int>& t) {
  std::printf("%d %d %d %d %d %d %d\n", std::get<0>(t), std::get<1>(t), std::get<2>(t), std::get<3>(t), std::get<4>(t),
              std::get<5>(t), std::get<6>(t));
}

int main() {
  int m, k, n, f32, gated, aligned;
  while (std::scanf("%d %d %d %d %d %d", &m, &k, &n, &f32, &gated, &aligned) == 6) print(kernel_of(m, k, n, f32, gated, aligned));
  std::puts("--");
  std::set<std::tuple<int, int, int, int, int, int, int>> all;
  std::mt19937_64 gen(17);
  const auto log = [&](double b) {
    return static_cast<int>(std::exp(std::uniform_real_distribution<double>(0.0, std::log(b))(gen)));
  };
  for (int i = 0; i < 2000000; ++i) {
    f32 = gen() % 2, gated = gen() % 2, aligned = gen() % 2;
    m = log(20000), n = log(40000), k = log(30000);
    if (aligned) k = (k + 7) / 8 * 8;
    all.insert(kernel_of(m, k, n, f32, gated, aligned));
  }
  for (const auto& t : all) print(t);
}
"""


def test_every_kernel_that_a_plan_gives_has_its_shape(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "plan"
    src.write_text(MAIN)
    subprocess.run([os.environ.get("CXX_HOST", "g++"), "-O2", "-std=c++17", f"-I{CSRC}", str(src),
                    os.path.join(CSRC, "tts_linear.cpp"), "-o", str(exe)], check=True, capture_output=True)
    lines = [f"{m} {k} {n} {int(t == 'f32')} {int(gated)} {int(aligned)}"
             for (t, gated, _, _, _, aligned, _), (m, k, n) in TILES.items()]
    r = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True, timeout=300, check=True)
    listed, found = ([tuple(map(int, x.split())) for x in part.strip().splitlines()] for part in r.stdout.split("--\n"))
    wanted = [(int(t == "f32"), *map(int, rest)) for t, *rest in TILES]
    moved = [(w, got, s) for w, got, s in zip(wanted, listed, TILES.values()) if w != got]
    assert not moved, f"(kernel, the one that the plan gives now, shape): {moved}"
    assert set(found) == set(wanted), (set(found) - set(wanted), set(wanted) - set(found))
