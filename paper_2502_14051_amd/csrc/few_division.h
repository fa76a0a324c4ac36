// How the attention of few rows over a quantised cache is divided between workgroups.  Plain arithmetic that needs no device,
// so a host program can sweep it.
//
// A workgroup fills a compute unit; its wavefronts take units of 32 keys in turn, and a round of them takes as long as memory
// does.  The keys of every tile of rows are cut into parts so that there are as many as compute units, but where a part
// would be less than a round, and not where two rounds would do: handing results over takes about what a round takes.
// (16 sequences' lists of 1024 tokens, 8 KV heads, us in one, two and four parts: 17.2, 18.8, 23.2; one sequence's of 2048
// in one, two, four and eight: 19.4, 16.8, 14.7, 14.1.)
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define RKV_HD __host__ __device__
#else
#define RKV_HD
#endif

namespace rkv {

constexpr int kFewRound = 16;  // units that a workgroup's wavefronts take at a time

// Parts of a tile that sees `units` units, at `share` parts to a unit.
RKV_HD inline int few_parts(int units, float share) {
  if (units <= 2 * kFewRound) return 1;
  const int n = (int)((float)units * share), most = units / kFewRound;
  return n < 1 ? 1 : n > most ? most : n;
}

// Parts to a unit.  `work`: units of all tiles, `tiles`: how many, `slots`: compute units; `count(share)`: parts of all tiles,
// which the result keeps within `slots` unless the tiles alone exceed it.
template <class Count>
RKV_HD inline float few_share(float work, int tiles, int slots, const Count& count) {
  if (tiles >= slots) return 0.f;
  float share = (float)slots / work * 1.000001f;  // (so that equal tiles get what they should in spite of rounding)
  for (int i = 0; i < 24; ++i) {
    const int n = count(share);
    if (n <= slots) return share;
    share *= (float)slots / (float)n * 0.98f;
  }
  return 0.f;
}

}  // namespace rkv
