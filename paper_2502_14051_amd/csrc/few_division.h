// How the attention of few rows over a quantised cache is divided between workgroups.  Plain arithmetic that needs no device,
// so a host program can sweep it.
//
// A workgroup fills a compute unit; its wavefronts take units of 32 keys in turn, and a round of them takes as long as memory
// does.  Where workgroups suffice, every tile is cut into parts of its own, a round each or what more of them are needed for all
// tiles; tiles of two rounds at most are whole, as handing results over takes about what a round takes.  (16 sequences' lists of
// 1024 tokens, 8 KV heads, us in one, two and four parts: 17.2, 18.8, 23.2; one sequence's of 2048 in one, two, four and eight:
// 19.4, 16.8, 14.7, 14.1.)
// (A token of each of 8 sequences of up to 5211, one KV head, 17.3 us so and 25.1 in equal pieces of all; of 16 of up to 3000, 8
// KV heads, 23.7 and 29.7: a workgroup whose piece holds the end of one tile and the beginning of another does both in turn.)
// Where that would leave workgroups idle, or they have many rounds to take, the units of all tiles of a KV head stand in a row,
// tile behind tile, and every workgroup takes an equal piece of it, wherever that begins and ends: lengths may differ as they
// like.  A tile that lies in several pieces has that many parts, whose results are joined; of a piece only the first and the
// last tile can be such.
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

// Parts of a tile of `units` units, `size` to a part at most.
RKV_HD inline int few_parts(int units, int size) { return units <= 2 * kFewRound ? 1 : units / size + (units % size != 0); }
// The sizes tried for them, `more` = 0, 1, ..: the fewest rounds that all units could do with, then a round more each.  Parts of
// size 0: pieces of the row instead.
constexpr int kFewTries = 2;
constexpr int kFewLong = 8;  // rounds to a workgroup from which on no size is tried (which takes 1 us)
RKV_HD inline int few_tries(int units, int slots) { return units / kFewLong / kFewRound <= slots ? kFewTries : 0; }
RKV_HD inline int few_size(int units, int slots, int more) {
  const int least = units / slots + (units % slots != 0);
  return (least < kFewRound ? kFewRound : least) + more * kFewRound;
}
// Pieces of a row of `units` units of `tiles` tiles, `slots` at most.
RKV_HD inline int few_pieces(int units, int tiles, int slots) {
  const int n = units / 2 / kFewRound <= tiles && units <= 2 * kFewRound * (int64_t)tiles ? tiles : units / kFewRound;
  return n > slots ? slots : n < 1 ? 1 : n;
}
// Pieces that either way makes at most.
RKV_HD inline int few_most(int units, int tiles, int slots) {
  const int64_t n = (int64_t)units / kFewRound + tiles;
  return n > slots ? slots : n < 1 ? 1 : (int)n;
}
// First unit of piece k of `pieces` (of piece `pieces`: the end): floor(units k / pieces), in 32 bits.
RKV_HD inline int few_begin(int units, int k, int pieces) {
  const uint32_t each = (uint32_t)units / (uint32_t)pieces, rest = (uint32_t)units - each * (uint32_t)pieces;
  return (int)(each * (uint32_t)k + rest * (uint32_t)k / (uint32_t)pieces);
}
// The piece that unit x lies in: the last that begins at x or before, begin(k) <= x being k < (x + 1) pieces / units.  Of long
// rows pieces have 2^16 units and more, so it is the one in which x would lie if all had one more, or the next.
RKV_HD inline int few_piece_of(int units, int x, int pieces) {
  if (units < (1 << 24)) return (int)(((uint32_t)(x + 1) * (uint32_t)pieces - 1u) / (uint32_t)units);
  const int k = (int)((uint32_t)x / ((uint32_t)units / (uint32_t)pieces + 1u));
  return k + (few_begin(units, k + 1, pieces) <= x);
}

// Units of all tiles at most: `rows` tokens of `batch` sequences in tiles of `tile_tokens`, of caches with room for `room` tokens.
// What a launch has places for, and 32 bits count.  It holds where the rows of the sequences add up to `rows` at most; rows that
// two sequences share (starts that do not ascend) can come to any number of units, so a launch that finds more does nothing.
RKV_HD inline int64_t few_bound(int rows, int batch, int tile_tokens, int64_t room) {
  const int64_t tiles = (int64_t)rows / tile_tokens + batch;
  return (tiles < rows ? tiles : rows) * ((room + 31) / 32);
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
