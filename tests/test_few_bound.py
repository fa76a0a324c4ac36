"""What a launch of the attention of few rows over a quantised cache is planned for, swept on the CPU from the header the kernels
include: rows that no two sequences share stay within it, others need not, and are told apart by their sum."""
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
static int ceil_of(int64_t a, int b) { return (int)((a + b - 1) / b); }
int main() {
  int bad = 0, over = 0, wrapped = 0;
  static int starts[9000];
  for (int trial = 0; trial < 40000 && bad < 10; ++trial) {
    const int B = 1 + rnd(trial % 7 == 0 ? 8192 : 20), tile_tokens = 1 + rnd(64), n = 1 + rnd(64 * B);
    const int64_t room = 1 + rnd(trial % 3 == 0 ? 1 << 30 : 5000);
    const bool ascend = trial % 2 == 0;
    for (int b = 0; b <= B; ++b) starts[b] = ascend ? (int)rnd(n + 1) : b % 2 ? n : 0;
    if (ascend)  // (an insertion sort)
      for (int i = 1; i <= B && B < 50; ++i)
        for (int j = i; j > 0 && starts[j] < starts[j - 1]; --j) { const int t = starts[j]; starts[j] = starts[j - 1]; starts[j - 1] = t; }
    if (ascend && B >= 50)
      for (int b = 0; b <= B; ++b) starts[b] = (int)((int64_t)n * b / B);
    int64_t rows = 0, units = 0;
    for (int b = 0; b < B; ++b) {
      const int own = starts[b + 1] > starts[b] ? starts[b + 1] - starts[b] : 0;
      rows += own;
      units += (int64_t)ceil_of(own, tile_tokens) * ceil_of(room, 32);  // of caches that are full
    }
    const int64_t bound = few_bound(n, B, tile_tokens, room);
    if (rows <= n && units > bound) { ++bad; printf("trial %d: %lld units of %lld\n", trial, (long long)units, (long long)bound); }
    if (ascend && rows > n) { ++bad; printf("trial %d: rows\n", trial); }
    over += rows > n && units > bound;
    wrapped += rows > n && bound < 1ll << 31 && units >= 1ll << 31;  // the piece of a workgroup could begin in front of the first tile
  }
  printf("%d over, %d beyond 32 bits\n", over, wrapped);
  return bad != 0 || over < 1000 || wrapped < 100;
}
"""


def test_what_is_planned_for(tmp_path):
    src, exe = tmp_path / "bound.cc", tmp_path / "bound"
    src.write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2502_14051_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I" + inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
