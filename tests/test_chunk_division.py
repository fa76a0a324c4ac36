"""How the attention of a chunk is divided, swept on the CPU from the header the kernels include: no more workgroups than
are launched, no part smaller than sensible, balance."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include "chunk_division.h"
using namespace rkv;
static uint64_t state = 88172645463325252ull;
static uint32_t rnd(uint32_t n) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (uint32_t)(state % n); }
int main() {
  int bad = 0, cut = 0;
  static int tiles[300], steps[300];
  for (int trial = 0; trial < 60000; ++trial) {
    const int slots = trial & 1 ? 256 : 512, B = 1 + rnd(trial % 3 == 0 ? 300 : 8), heads = 1 + rnd(16);
    const int most_tiles = 1 + rnd(trial % 5 == 0 ? 200 : 4), longest = 1 + rnd(trial % 4 == 0 ? 30000 : 600);
    ChunkLoad load = {0, 0.f, 0};
    for (int b = 0; b < B; ++b) {
      tiles[b] = rnd(most_tiles + 1);
      steps[b] = tiles[b] ? 1 + rnd(longest) : 0;
      load.tiles += tiles[b] * heads;
      load.work += (float)tiles[b] * (float)steps[b] * (float)heads;
      if (steps[b] > load.longest) load.longest = steps[b];
    }
    const auto count = [&](int size) {
      int64_t n = 0;
      for (int b = 0; b < B; ++b) n += (int64_t)tiles[b] * chunk_parts(steps[b], size);
      return (int)(n * heads);
    };
    const int most = slots * chunk_rounds(trial % 7 ? load.tiles : rnd(load.tiles + 1), slots);
    const int size = chunk_part_size(load, slots, most, count), n = count(size);
    const int launched = load.tiles > most ? load.tiles : most;
    if (n > launched) { ++bad; printf("trial %d: %d workgroups, %d launched\n", trial, n, launched); }
    if (size != kChunkWhole) {
      ++cut;
      if (n > most) { ++bad; printf("trial %d: parts without a place\n", trial); }
      if (size < kChunkLeastSteps) { ++bad; printf("trial %d: parts of %d steps\n", trial, size); }
      if (load.tiles >= most) { ++bad; printf("trial %d: cut without need\n", trial); }
    } else if (n != load.tiles) { ++bad; printf("trial %d: whole tiles in parts\n", trial); }
    // a tile's parts cover its steps once, in order
    for (int b = 0; b < B && b < 4; ++b) {
      const int parts = chunk_parts(steps[b], size);
      const int seen = steps[b] ? 1 + rnd(steps[b]) : 0, per = chunk_ceil(seen, parts);
      int at = 0;
      for (int p = 0; p < parts; ++p) {
        const int it0 = p * per < seen ? p * per : seen, it1 = it0 + per < seen ? it0 + per : seen;
        if (it0 != at) { ++bad; printf("trial %d: a gap\n", trial); }
        at = it1;
      }
      if (at != seen) { ++bad; printf("trial %d: steps left over\n", trial); }
    }
    if (bad > 10) break;
  }
  // one long sequence fills the chip
  for (int tiles1 = 1; tiles1 <= 256; ++tiles1) {
    const int steps1 = 4000;
    ChunkLoad load = {tiles1, (float)tiles1 * steps1, steps1};
    const auto count = [&](int size) { return tiles1 * chunk_parts(steps1, size); };
    const int size = chunk_part_size(load, 256, 256 * chunk_rounds(tiles1, 256), count), n = count(size);
    const double rounds = chunk_ceil(n, 256), ideal = (double)tiles1 * steps1 / 256, took = rounds * chunk_ceil(steps1, chunk_parts(steps1, size));
    if (took > 1.5 * ideal + kChunkLeastSteps) { ++bad; printf("%d tiles: %.0f steps, ideal %.0f\n", tiles1, took, ideal); }
  }
  printf("%d cut, %d wrong\n", cut, bad);
  return bad || !cut;
}
"""


def test_sweep(tmp_path):
    src, exe = tmp_path / "sweep.cpp", tmp_path / "sweep"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I" + os.path.join(ROOT, "paper_2502_14051_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
