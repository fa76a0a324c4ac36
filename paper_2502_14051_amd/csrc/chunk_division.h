// How the attention of a chunk of new tokens is divided between workgroups.  Plain arithmetic that needs no device, so a
// host program can sweep it.
//
// The rows of a (sequence, KV head) are cut into tiles of whole tokens; a tile walks the keys its last token sees, a step
// at a time.  Where the tiles alone would leave compute units idle, the keys of every tile are cut as well and the parts
// are merged by a second launch.  A part is not free: its rows' sums go to memory and come back, and it begins with steps
// that overlap nothing; together what kChunkPartSteps steps of its work take.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define RKV_HD __host__ __device__
#else
#define RKV_HD
#endif

namespace rkv {

constexpr int kChunkPartSteps = 6;
constexpr int kChunkLeastSteps = 8;     // no part is smaller
constexpr int kChunkRounds = 3;         // parts for up to so many rounds of workgroups over the chip
constexpr int kChunkWhole = 1 << 30;    // nothing is cut

RKV_HD constexpr int chunk_ceil(int a, int b) { return a / b + (a % b != 0); }

// parts of a tile that sees `steps` steps, at `size` steps to a part
RKV_HD constexpr int chunk_parts(int steps, int size) { return steps <= size ? 1 : chunk_ceil(steps, size); }

struct ChunkLoad {
  int tiles;    // row tiles of all sequences and KV heads
  float work;   // steps of all of them
  int longest;  // steps of the longest
};

// Steps per part.  `slots`: workgroups the chip holds at a time; `count(size)`: workgroups at that size.  Of one to three
// rounds the best is taken: 56 tiles of 2049 steps over 256 slots come as 4 parts each in one round, 87 % of it, or as 9 in
// two, 98 %; 171 to 192 tiles gain nothing by halves in two rounds, but by quarters in three.  The result never needs more
// than max(tiles, slots * kChunkRounds) workgroups.
template <class Count>
RKV_HD inline int chunk_part_size(const ChunkLoad& load, int slots, const Count& count) {
  if (load.tiles >= slots * kChunkRounds || load.longest <= kChunkLeastSteps) return kChunkWhole;
  int best = kChunkWhole;
  int64_t cost = (int64_t)chunk_ceil(load.tiles, slots) * load.longest;
  for (int rounds = 1; rounds <= kChunkRounds; ++rounds) {
    const int most = slots * rounds;
    if (load.tiles >= most) continue;
    int size = (int)(load.work / (float)most);
    if (size < kChunkLeastSteps) size = kChunkLeastSteps;
    int n = count(size);
    while (n > most && size < load.longest) {
      size += size / 16 + 1;
      n = count(size);
    }
    if (size >= load.longest) continue;
    const int64_t c = (int64_t)chunk_ceil(n, slots) * (size + kChunkPartSteps);
    if (c < cost) {
      cost = c;
      best = size;
    }
  }
  return best;
}

}  // namespace rkv
