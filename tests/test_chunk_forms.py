"""Which form the attention of a chunk takes, by the header that the library includes (no GPU): the cases that test a form on
the GPU are the ones that take it, also after a rule has moved."""
import os
import subprocess

import pytest

import test_gpu_chunk_attend as narrow
import test_gpu_chunk_wide as wide

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "chunk_division.h"
using namespace rkv;
// far group heads room n {new len}: rows of a tile, past the caches, what is launched for parts (0: keys are not cut), parts, tiles
int main(int argc, char** argv) {
  const auto arg = [&](int i) { return atoll(argv[i]); };
  const bool far = arg(1) != 0;
  const int group = (int)arg(2), heads = (int)arg(3), n = (int)arg(5);
  const int64_t room = arg(4), held = (int64_t)n * room * heads * 128 * 2 * 2;
  int64_t rows_in = arg(6);  // rows of the packed tensors
  const int64_t rows = rows_in * group / n;
  const int tile_rows = chunk_tile_rows(far, rows, held), tok = tile_rows / group, slots = 256 * (256 / tile_rows);
  const int most = slots * chunk_rounds((rows_in + tok - 1) / tok * heads, slots);
  ChunkLoad load = {0, 0.f, 0};
  const auto each = [&](const auto& fn) {
    for (int b = 0; b < n; ++b) {
      const int t = chunk_ceil((int)arg(7 + 2 * b), tok);
      fn(t, t ? chunk_ceil((int)arg(8 + 2 * b), 64) : 0);
    }
  };
  each([&](int t, int steps) {
    load.tiles += t * heads;
    load.work += (float)t * (float)steps * (float)heads;
    if (steps > load.longest) load.longest = steps;
  });
  const auto count = [&](int size) {
    int k = 0;
    each([&](int t, int steps) { k += t * chunk_parts(steps, size); });
    return k * heads;
  };
  const int size = chunk_part_size(load, slots, most, count);
  printf("%d %d %d %d %d\n", tile_rows, (int)chunk_past_caches(far, rows, held), most, size == kChunkWhole ? 0 : count(size), load.tiles);
}
"""


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "form.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I" + os.path.join(ROOT, "paper_2502_14051_amd", "csrc"), str(d / "form.cpp"),
                    "-o", str(d / "form")], check=True)

    def ask(lens, news, hq, hkv, room, pad=0, far=False):
        args = [int(far), hq // hkv, hkv, room, len(lens), sum(news) + pad] + [x for b in range(len(lens)) for x in (news[b], lens[b])]
        r = subprocess.run([str(d / "form")] + [str(a) for a in args], capture_output=True, text=True, check=True)
        return tuple(int(x) for x in r.stdout.split())

    return ask


def room(lens, ps, spare_pages):
    return ((max(lens) + ps - 1) // ps + spare_pages + 7) // 8 * 8 * ps


@pytest.mark.parametrize("ps", [16, 3, 64])
def test_wide_tiles(form, ps):
    """Keys cut for one round of workgroups and for three, tiles whole though there is room for parts, and too many for that."""
    seen = {}
    for name, (lens, news, hq, hkv, tokens) in wide.CASES.items():
        rows, past, most, parts, tiles = form(lens, news, hq, hkv, room(lens, ps, (tokens - max(lens)) // ps), pad=3)
        assert rows == 256 and not past, name
        seen[name] = (most, parts, tiles)
    assert seen["one round"][0] == 256 and 0 < seen["one round"][2] < seen["one round"][1] <= 256
    assert seen["three rounds"][0] == 768 and seen["three rounds"][2] < seen["three rounds"][1] <= 768
    assert seen["not cut"][1] == 0 and seen["not cut"][2] >= 768
    assert 256 < seen["between"][2] < 768
    assert seen["ragged"][1] > 0


def test_wide_tiles_of_64_bit_offsets(form):
    cut = [form(lens, news, 32, 8, room(lens, 16, 0), far=True) for lens, news in wide.FAR_CASES]
    assert all(f[0] == 256 and not f[1] for f in cut) and cut[0][3] > 0 and cut[1][3] > 0 and cut[2][4] > 256
    assert wide.FAR_PAGES * 8 * 16 * 128 * 2 >= 1 << 32


def test_reading_past_the_caches(form):
    """And the short tiles of the other cases over small caches."""
    for ps in (16, 4):
        assert form([700, 5000, 1], [3, 20, 1], 8, 2, room([5000], ps, 100000 // ps))[:2] == (128, 1)
    assert form([9000], [70], 4, 1, room([9000], 16, 0))[:2] == (128, 0)
    assert narrow.pytestmark.name == "gpu"
