"""How the attention of few rows over a quantised cache is divided, swept on the CPU from the header the kernels include: pieces
that cover all units once and evenly, places for what they hand over."""
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
  int bad = 0, cut = 0, crossing = 0;
  static int tiles[300], units[300], begin[4000], end[4000];
  for (int trial = 0; trial < 60000 && bad < 10; ++trial) {
    const int slots = 1 + rnd(256), B = 1 + rnd(trial % 3 == 0 ? 300 : 8), most_tiles = 1 + rnd(trial % 5 == 0 ? 12 : 2);
    const int longest = trial % 9 == 0 ? 1 << 21 : 1 + rnd(trial % 4 == 0 ? 60000 : 600);
    int64_t all = 0, sum = 0;
    int n = 0;
    for (int b = 0; b < B; ++b) {
      tiles[b] = trial % 11 == 0 ? 1 : rnd(most_tiles + 1);
      units[b] = trial % 6 == 0 ? longest : 1 + rnd(longest);
      for (int t = 0; t < tiles[b]; ++t) {
        begin[n] = (int)sum;
        sum += units[b];
        end[n++] = (int)sum;
        if (sum >= 1ll << 31) break;
      }
      if (sum >= 1ll << 31) break;
      all += tiles[b];
    }
    if (sum >= 1ll << 31 || n == 0) continue;
    const int U = (int)sum, pieces = few_pieces(U, (int)all, slots);
    if (pieces < 1 || pieces > slots) { ++bad; printf("trial %d: %d pieces for %d\n", trial, pieces, slots); }
    if (pieces > 1 && U / pieces < kFewRound && U > 2 * kFewRound * all) { ++bad; printf("trial %d: short pieces\n", trial); }
    if (few_begin(U, 0, pieces) != 0 || few_begin(U, pieces, pieces) != U) { ++bad; printf("trial %d: ends\n", trial); }
    for (int k = 0; k < pieces; ++k) {
      const int x0 = few_begin(U, k, pieces), x1 = few_begin(U, k + 1, pieces);
      if (x0 != (int)((int64_t)U * k / pieces)) { ++bad; printf("trial %d: piece %d begins at %d\n", trial, k, x0); }
      if (x1 - x0 > U / pieces + 1 || x1 - x0 < U / pieces) { ++bad; printf("trial %d: uneven\n", trial); }
      if (x1 > x0 && (few_piece_of(U, x0, pieces) != k || few_piece_of(U, x1 - 1, pieces) != k)) { ++bad; printf("trial %d: piece %d\n", trial, k); }
    }
    // a piece's places: at most one tile begins in it and goes on, at most one goes on in it
    static int goes_on[300], went_on[300];
    for (int k = 0; k < pieces; ++k) goes_on[k] = went_on[k] = 0;
    for (int t = 0; t < n; ++t) {
      const int f = few_piece_of(U, begin[t], pieces), l = few_piece_of(U, end[t] - 1, pieces);
      if (l > f) {
        ++cut;
        ++goes_on[f];
        for (int k = f + 1; k <= l; ++k) ++went_on[k];
      } else if (f > 0 && begin[t] > few_begin(U, f, pieces)) ++crossing;
    }
    for (int k = 0; k < pieces; ++k)
      if (goes_on[k] > 1 || went_on[k] > 1) { ++bad; printf("trial %d: piece %d has no place\n", trial, k); }
  }
  // parts of tiles that nothing else shares
  int whole = 0, own = 0, fits[2] = {0, 0};
  for (int trial = 0; trial < 40000 && bad < 10; ++trial) {
    const int slots = 1 + rnd(256), n = 1 + rnd(trial % 2 ? 300 : 12), longest = 1 + rnd(trial % 4 == 0 ? 60000 : trial % 3 == 0 ? 60 : 600);
    int sum = 0;
    for (int t = 0; t < n; ++t) sum += units[t] = 1 + (trial % 5 == 0 ? longest - 1 : rnd(longest));
    for (int i = 0; i < kFewTries; ++i) {
      const int size = few_size(sum, slots, i);
      if (size < kFewRound || (int64_t)size * slots < sum) { ++bad; printf("trial %d: size %d\n", trial, size); }
      int64_t parts = 0;
      for (int t = 0; t < n; ++t) parts += few_parts(units[t], size);
      if (parts > slots) continue;
      ++fits[i];
      if (parts > few_most(sum, n, 256)) { ++bad; printf("trial %d: %d parts\n", trial, (int)parts); }
      for (int t = 0; t < n; ++t) {
        const int k = few_parts(units[t], size);
        ++(k == 1 ? whole : own);
        for (int j = 0; j < k; ++j) {
          const int len = few_begin(units[t], j + 1, k) - few_begin(units[t], j, k);
          if (len < 1 || (k > 1 && len > size)) { ++bad; printf("trial %d: part of %d\n", trial, len); }
        }
        if (few_begin(units[t], 0, k) != 0 || few_begin(units[t], k, k) != units[t]) { ++bad; printf("trial %d: ends of parts\n", trial); }
      }
      break;
    }
  }
  if (whole < 5000 || own < 5000 || fits[0] < 1000 || fits[1] < 1000) { ++bad; printf("%d whole, %d cut, sizes %d %d\n", whole, own, fits[0], fits[1]); }
  // equal tiles: as many pieces to each as fit, none across two
  for (int t = 1; t <= 32; t *= 2) {
    const int pieces = few_pieces(t * 129, t, 32);
    for (int k = 0; k < 32; ++k)
      if (pieces != (t == 1 ? 8 : t == 2 ? 16 : 32) || (t > 2 && few_begin(t * 129, k * 32 / t, pieces) % 129 && k * 32 / t < 32 && k < t)) { ++bad; printf("%d tiles: %d pieces\n", t, pieces); break; }
  }
  for (int d = 1; d <= 64; ++d)
    for (int i = 0; i < 200000; ++i) {
      const uint32_t n = i < 3000 ? i : i < 6000 ? 0x7fffffffu - (i - 3000) : i < 100000 ? rnd(0x80000000u) : (uint32_t)d * rnd(0x7fffffffu / d) - (i & 1);
      if (n < 0x80000000u && divide(n, divider(d)) != n / d) { ++bad; printf("%u / %d\n", n, d); break; }
    }
  printf("%d cut, %d whole beside others\n", cut, crossing);
  return bad != 0 || cut < 5000 || crossing < 5000;
}
"""


def test_division(tmp_path):
    src, exe = tmp_path / "sweep.cc", tmp_path / "sweep"
    src.write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2502_14051_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I" + inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
