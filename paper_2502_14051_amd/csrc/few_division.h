// How the attention of few rows over a quantised cache is divided between workgroups.  Plain arithmetic that needs no device,
// so a host program can sweep it.
//
// A workgroup fills a compute unit; its wavefronts take units of 32 keys in turn, and a round of them takes as long as memory
// does.  The units of all tiles of a KV head stand in a row, tile behind tile, and every workgroup takes an equal piece of it,
// wherever that begins and ends: lengths may differ as they like.  A tile that lies in several pieces has that many parts,
// whose results are joined; of a piece only the first and the last tile can be such.
// No piece is shorter than a round, and where tiles have two rounds at most they are whole as far as workgroups suffice:
// handing results over takes about what a round takes.  (16 sequences' lists of 1024 tokens, 8 KV heads, us in one, two and
// four parts: 17.2, 18.8, 23.2; one sequence's of 2048 in one, two, four and eight: 19.4, 16.8, 14.7, 14.1.)
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define RKV_HD __host__ __device__
#else
#define RKV_HD
#endif

namespace rkv {

constexpr int kFewMost = 256;  // pieces at most
constexpr int kFewRound = 16;  // units that a workgroup's wavefronts take at a time

// Pieces of a row of `units` units of `tiles` tiles, `slots` at most.
RKV_HD inline int few_pieces(int units, int tiles, int slots) {
  const int n = units / 2 / kFewRound <= tiles && units <= 2 * kFewRound * (int64_t)tiles ? tiles : units / kFewRound;
  return n > slots ? slots : n < 1 ? 1 : n;
}
// First unit of piece k (of piece `pieces`: the end).  (Most rows are short enough for 32 bits, whose division is the shorter.)
RKV_HD inline int few_begin(int units, int k, int pieces) {
  if (units < (1 << 24)) return (int)((uint32_t)units * (uint32_t)k / (uint32_t)pieces);
  return (int)((uint64_t)units * (uint64_t)k / (uint32_t)pieces);
}
// The piece that unit x lies in: the last that begins at x or before, begin(k) <= x being k < (x + 1) pieces / units.
RKV_HD inline int few_piece_of(int units, int x, int pieces) {
  if (units < (1 << 24)) return (int)(((uint32_t)(x + 1) * (uint32_t)pieces - 1u) / (uint32_t)units);
  return (int)(((uint64_t)(x + 1) * (uint64_t)pieces - 1u) / (uint32_t)units);
}

// Division of numbers below 2^31 by the same one again and again: n / d = (hi(n m) + n) >> l with l = ceil(log2 d) and
// m = floor(2^32 (2^l - d) / d) + 1 (Granlund and Montgomery 1994).
struct Divider {
  uint32_t m;
  int32_t l;
};
inline Divider divider(int d) {
  int l = 0;
  while ((1 << l) < d) ++l;
  return {(uint32_t)(((((uint64_t)1 << l) - (uint64_t)d) << 32) / (uint64_t)d + 1u), l};
}
RKV_HD inline uint32_t divide(uint32_t n, Divider by) { return ((uint32_t)(((uint64_t)n * by.m) >> 32) + n) >> by.l; }

}  // namespace rkv
