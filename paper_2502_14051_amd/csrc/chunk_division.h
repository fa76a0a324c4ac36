// How the attention of a chunk of new tokens is divided between workgroups.  Plain arithmetic that needs no device, so a
// host program can sweep it.
//
// The rows of a (sequence, KV head) are cut into tiles of whole tokens; a tile walks the keys its last token sees, `step`
// of them at a time.  Where the tiles alone would leave compute units idle, the keys of every tile are cut as well and
// the parts are merged by a second launch.  A part is not free: its rows' sums go to memory and come back (a 256-row tile
// 266 KB, what four steps of its work take), so parts hold at least kChunkLeastSteps steps.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define RKV_HD __host__ __device__
#else
#define RKV_HD
#endif

namespace rkv {

constexpr int kChunkLeastSteps = 8;

RKV_HD constexpr int chunk_ceil(int a, int b) { return (int)(((int64_t)a + b - 1) / b); }

// parts of a tile that sees `steps` steps, at `size` steps to a part
RKV_HD constexpr int chunk_parts(int steps, int size) { return steps <= size ? 1 : chunk_ceil(steps, size); }

// Steps per part.  `tiles`: row tiles of all sequences and KV heads; `work`: steps of all of them; `target`: workgroups
// wanted; `count(size)`: workgroups at that size.  The result never needs more than max(tiles, target) workgroups.
constexpr int kChunkWhole = 1 << 30;  // nothing is cut
template <class Count>
RKV_HD inline int chunk_part_size(int64_t tiles, int64_t work, int target, int longest, const Count& count) {
  if (tiles >= target) return kChunkWhole;
  int64_t size = (work + target - 1) / target;
  if (size < kChunkLeastSteps) size = kChunkLeastSteps;
  while (size < longest && count((int)size) > target) size += size / 16 + 1;
  return size < longest ? (int)size : kChunkWhole;
}

}  // namespace rkv
