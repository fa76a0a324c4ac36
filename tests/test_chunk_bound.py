"""The division of a chunk's attention where sequences share rows (starts that do not ascend), on the CPU from the header that the
kernels include: however many tiles they come to, nothing is cut into more parts than there are places for."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdint.h>
#include <stdio.h>
#include "chunk_division.h"
using namespace rkv;
static uint64_t state = 88172645463325252ull;
static uint32_t rnd(uint32_t n) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (uint32_t)(state % n); }
int main() {
  int bad = 0, many = 0, wrapped = 0, cut = 0;
  for (int trial = 0; trial < 20000 && bad < 10; ++trial) {
    const bool round = trial % 4 == 1;  // as many tiles as 32 bits come to, and a few more of the first sequence
    const int heads = round ? 1 : 1 << rnd(5), B = round ? 8192 : 1 + rnd(8192 / heads), tile_rows = rnd(2) ? 128 : 256, slots = 256 * (256 / tile_rows);
    const int most = slots * (rnd(2) ? kChunkRounds : 1), steps = 1 + rnd(trial % 2 ? 1 << 24 : 2000);
    const int tiles = round ? 1 << 19 : trial % 3 ? 1 + rnd(1 << 21) : rnd(3);  // of each sequence; all of the same length
    const int more = round ? 1 + rnd(most) : 0;
    const auto in32 = [](int64_t x) { return (int)(uint32_t)(uint64_t)x; };
    const auto count = [&](int size) { return in32(((int64_t)B * tiles + more) * chunk_parts(steps, size) * heads); };  // as 32 bits have it
    ChunkLoad load = {0, 0.f, steps};
    for (int b = 0; b < B; b += 64)  // a wavefront's lanes in 32 bits, wavefront by wavefront in fp32
      load.work += (float)in32((int64_t)(B - b < 64 ? B - b : 64) * (tiles < most ? tiles : most) * (steps < 1 << 15 ? steps : 1 << 15)) * (float)heads;
    for (int b = 0; b < B; b += 64) load.tiles = chunk_add_tiles(load.tiles, (B - b < 64 ? B - b : 64) * tiles + (b == 0 ? more : 0), heads, most);
    const int64_t all = ((int64_t)B * tiles + more) * heads;
    if (load.tiles != (all < most ? all : most)) { ++bad; printf("trial %d: %d tiles of %lld\n", trial, load.tiles, (long long)all); }
    const int size = chunk_part_size(load, slots, most, count);
    const int64_t parts = all * chunk_parts(steps, size);
    if (size != kChunkWhole && parts > most) { ++bad; printf("trial %d: %lld parts, places for %d\n", trial, (long long)parts, most); }
    cut += size != kChunkWhole;
    many += all >= 1ll << 31;
    ChunkLoad old = {in32(all), load.work, steps};  // a count that has wrapped
    if (all > most) wrapped += chunk_part_size(old, slots, most, count) != kChunkWhole;
  }
  printf("%d of many tiles, %d would have been cut, %d are\n", many, wrapped, cut);
  return bad != 0 || many < 100 || wrapped < 10 || cut < 10;
}
"""


def test_parts_have_places(tmp_path):
    src, exe = tmp_path / "bound.cc", tmp_path / "bound"
    src.write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2502_14051_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I" + inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
