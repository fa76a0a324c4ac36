"""How the attention of few rows over a quantised cache is divided, swept on the CPU from the header the kernels include: no
more parts than workgroups are launched, none shorter than a round, all units covered once."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdint.h>
#include <stdio.h>
#include "few_division.h"
using namespace rkv;
static uint64_t state = 88172645463325252ull;
static uint32_t rnd(uint32_t n) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (uint32_t)(state % n); }
int main() {
  int bad = 0, cut = 0;
  static int tiles[300], units[300];
  for (int trial = 0; trial < 60000; ++trial) {
    const int slots = trial & 1 ? 256 : 512, B = 1 + rnd(trial % 3 == 0 ? 300 : 8), heads = 1 + rnd(16);
    const int most_tiles = 1 + rnd(trial % 5 == 0 ? 40 : 2), longest = 1 + rnd(trial % 4 == 0 ? 60000 : 600);
    int all = 0;
    float work = 0.f;
    for (int b = 0; b < B; ++b) {
      tiles[b] = trial % 11 == 0 ? 1 : rnd(most_tiles + 1);
      units[b] = tiles[b] ? trial % 6 == 0 ? longest : rnd(longest + 1) : 0;
      all += tiles[b] * heads;
      work += (float)tiles[b] * (float)units[b] * (float)heads;
    }
    const auto count = [&](float share) {
      int64_t n = 0;
      for (int b = 0; b < B; ++b) n += (int64_t)tiles[b] * few_parts(units[b], share);
      return (int)(n * heads);
    };
    const float share = few_share(work, all, slots, count);
    const int n = count(share);
    if (n > (all > slots ? all : slots)) { ++bad; printf("trial %d: %d parts, %d tiles\n", trial, n, all); }
    if (all >= slots && n != all) { ++bad; printf("trial %d: cut without need\n", trial); }
    cut += n > all;
    for (int b = 0; b < B; ++b) {
      const int parts = few_parts(units[b], share);
      if (parts > 1 && units[b] / parts < kFewRound) { ++bad; printf("trial %d: %d units in %d parts\n", trial, units[b], parts); }
      int at = 0;
      for (int p = 0; p < parts; ++p) {
        const int u0 = (int)((int64_t)units[b] * p / parts), u1 = (int)((int64_t)units[b] * (p + 1) / parts);
        if (u0 != at || u1 < u0) { ++bad; printf("trial %d: a gap\n", trial); }
        at = u1;
      }
      if (at != units[b]) { ++bad; printf("trial %d: units left over\n", trial); }
    }
    if (bad > 10) break;
  }
  // equal tiles of many units fill the chip as far as whole parts do
  for (int t = 1; t < 256; ++t)
    for (int u = 600; u < 20000; u += 777) {
      const auto count = [&](float s) { return t * few_parts(u, s); };
      const int n = count(few_share((float)t * (float)u, t, 256, count)), want = 256 / t < u / kFewRound ? 256 / t : u / kFewRound;
      if (n != t * want) { ++bad; printf("%d tiles of %d units: %d parts\n", t, u, n); break; }
    }
  printf("%d cut\n", cut);
  return bad != 0 || cut < 5000;
}
"""


def test_division(tmp_path):
    src, exe = tmp_path / "sweep.cc", tmp_path / "sweep"
    src.write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2502_14051_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I" + inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
