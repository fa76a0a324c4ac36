// How the attention of a chunk of new tokens is divided between workgroups.  Plain arithmetic that needs no device, so a
// host program can sweep it.
//
// The rows of a (sequence, KV head) are cut into tiles of whole tokens; a tile walks the keys its last token sees, a step
// at a time.  Where the tiles alone would leave compute units idle, the keys of every tile are cut as well and the parts
// are merged by a second launch.  A part is not free: its rows' sums go to memory and come back, and it begins with steps
// that overlap nothing; together what kChunkPartSteps steps of its work take.
// (For a prompt alone, whose last tile sees twice the mean, parts of the long tiles only were no gain either: 2048 tokens
// 80 us so, 62 whole.)
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define RKV_HD __host__ __device__
#else
#define RKV_HD
#endif

namespace rkv {

constexpr int kChunkPartSteps = 8;
constexpr int kChunkLeastSteps = 4;     // no part is smaller
constexpr int kChunkShort = kChunkLeastSteps + kChunkPartSteps;  // a part of the least size costs what so short a tile does
constexpr int kChunkRounds = 3;         // parts for up to so many rounds of workgroups over the chip, see chunk_rounds
constexpr int kChunkWhole = 1 << 30;    // nothing is cut

RKV_HD constexpr int chunk_ceil(int a, int b) { return a / b + (a % b != 0); }

// parts of a tile that sees `steps` steps, at `size` steps to a part
RKV_HD constexpr int chunk_parts(int steps, int size) { return steps <= size ? 1 : chunk_ceil(steps, size); }

struct ChunkLoad {
  int tiles;    // row tiles of all sequences and KV heads, see chunk_add_tiles
  float work;   // steps of all of them
  int longest;  // steps of the longest
};

// Rounds of workgroups that parts are made for.  One, where tiles are few: a second round's finer parts gain less than its
// workgroups cost, most of them with nothing to do where few keys leave few parts (measured over 24 shapes: 2 % slower on
// average, 10 % at most).  From half as many tiles as slots on, one round has no room to cut, and 129 to 255 tiles would
// leave up to half of the chip idle: three, so that 192 tiles come as quarters.
RKV_HD constexpr int chunk_rounds(int64_t tiles, int slots) { return 2 * tiles > slots ? kChunkRounds : 1; }

// `tiles` and `more` of each of `heads`, counted up to `most`, from which on nothing is cut.  (Sequences whose rows overlap, of
// starts that do not ascend, can come to more than 32 bits count; a count that had wrapped would cut keys into parts that the
// merge looks for behind the end of the workspace.)
RKV_HD constexpr int chunk_add_tiles(int tiles, int more, int heads, int most) {
  return tiles + (int64_t)more * heads < most ? tiles + more * heads : most;
}

// Steps per part.  `slots`: workgroups the chip holds at a time, `most`: a multiple of it that the result does not exceed
// unless the tiles do; `count(size)`: workgroups at that size.
template <class Count>
RKV_HD inline int chunk_part_size(const ChunkLoad& load, int slots, int most, const Count& count) {
  if (load.tiles >= most || load.longest <= kChunkShort) return kChunkWhole;
  int best = kChunkWhole;
  int64_t cost = (int64_t)chunk_ceil(load.tiles, slots) * load.longest;
  for (int limit = slots; limit <= most; limit += slots) {
    if (load.tiles >= limit) continue;
    int size = (int)(load.work / (float)limit);
    if (size < kChunkLeastSteps) size = kChunkLeastSteps;
    int n = count(size);
    while (n > limit && size < load.longest) {
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

// Rows of a tile.  `far`: offsets of 64 bits, `rows`: of a sequence on average, `held`: bytes of keys and values there is
// room for.  128 rows to a workgroup, two of which run beside each other out of step, or 256, which share what is read.  The
// second reading of the keys costs where many tiles read keys that the caches do not hold (us with 128 rows and with 256,
// 32 heads over 8): 387 tokens behind 131072 (514 MiB) 1043 and 946, behind 65536 501 and 441, 2048 behind 131072 4289 and
// 4199, prompts of up to 16384 (192 MiB) 3325 and 3252.  Where they hold them or few tiles read, the finer tiles gain: a
// prompt of 2048 61.1 and 65.7, 2048 behind 6144 250 and 256, two prompts of up to 4096 198 and 206, 160 tokens behind 40960
// (161 MiB) 125 and 133.  From 64 to 160 MiB it makes no difference (2048 behind 24576 817 and 817, behind 32768 1064 and
// 1067).  With 64-bit offsets the registers of the former do not suffice.
RKV_HD constexpr int chunk_tile_rows(bool far, int64_t rows, int64_t held) { return !far && (rows <= 512 || held <= 128ll << 20) ? 128 : 256; }

// Keys that one tile reads, of caches that the 256 MiB of the last-level cache do not keep until the next call, are read
// past the caches: 5 tokens of each of 16 sequences of up to 32768 take 185 us so, 211 without; but 16 tokens behind 4000,
// called again at once, 17.8, without 16.5, and where several tiles read the same keys (387 tokens behind 131072, 256 rows
// to a tile) 1061, without 946.
RKV_HD constexpr bool chunk_past_caches(bool far, int64_t rows, int64_t held) { return rows <= 128 && !far && held > 256ll << 20; }

}  // namespace rkv
