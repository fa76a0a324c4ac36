// Causal attention of a chunk of new tokens over the paged cache they have been put into: whole prompts, the next piece
// of a prompt, a turn, drafted tokens, single tokens, in any mixture.
//
// Rows of a (sequence, KV head) are its new tokens times the group's query heads, so every key serves the whole group.
// A workgroup takes a tile of rows, 32 to a wavefront, and walks the keys 64 at a time through LDS, one pass with
// the running maximum m and sum l of each row:
//
//   S^T[key][row]     = K[key][:] . Q[row][:]              A = keys (32 rows), B = queries, kept in registers
//   O^T[chan][row]   += V^T[chan][key] . P^T[key][row]     A = values by channel, B = exp2(S c - m)
//
// Both products have the row as their column, so a lane owns one row: its 16 logits of a product, maximum, sum and
// outputs never leave it, but for one exchange with the lane 32 further, which holds the same row's other keys.  The
// product leaves a lane the keys of A's rows 8a + 4h + r; with the rows of K read in an order that swaps bits 2 and 3,
// these are keys 16x + 8h + 0..7, which packed to bf16 are the second product's operand as they stand.  P is rounded to
// bf16 there (relative 2^-8 at most each; fp32 operands would run at a sixteenth of the matrix rate); everything else is fp32.
//
// What that rounding costs is mostly the rows that few keys dominate: their weight's error is the result's.  It cancels where
// the result is divided by the sum of the rounded weights.  So a row has two sums, l of the weights as they are, which the
// log sum-exp takes, and lr, in which a unit of keys that outweighs all before it (kept apart for the lane's half of the keys)
// counts as rounded.  Relative to 64 bits, over all outputs, the cases of 5 to 8191 new tokens are off by 0.0019 to 0.0021 so,
// by 0.0022 to 0.0023 with l alone, by 0.0017 if the result alone is rounded.  That takes 0 to 2 % of their time (2048 tokens
// behind 32768 1048 and 1058 us, 6 prompts of up to 8191 1465 and 1490) and 5 % where keys are cut short (100 tokens of each of
// 2 sequences of 8000, 54.4 and 57.1); every unit counted as rounded is no better (0.0019 to 0.0021) and took 6 to 10 %.
//
// What bounds it.  Many rows: the matrix cores and, beside them, the vector instructions of the exponentials, at the clock
// that the chip's power leaves (2.0 GHz).  2048 tokens of 32 heads behind 32768, 8 KV heads, take 1.04 to 1.12 ms, 1.01 to
// 1.09 PFLOP/s, the matrix cores busy 52 % of the cycles; without loads and LDS reads the same instructions ran at 1.30, a
// library's product of 8192^3 runs at 1.40.  Few rows: HBM, 6.2 TB/s for 5 tokens of each of 16 sequences of up to 32768.
// Why 32 rows to a wavefront and two wavefronts to a SIMD: one stands at its products while the other forms exponentials.
// 64 rows, one wavefront to a SIMD, would read keys and values half as often, but its sums then travel between the two
// register files every step: 0.65 PFLOP/s; the two wavefronts alternating by barriers 0.62 to 0.87; products and
// exponentials of one unit one after the other 0.92; with the next unit's operands requested ahead 0.97; exponentials
// beside the products, fenced so that they stay there, 1.05; and with a raised priority while they do, 1.09.
#include <type_traits>

#include "attend_core.h"
#include "chunk_division.h"

namespace rkv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;                                        // keys per step
constexpr int kKeyBytes = kStep * kHeadDim * (int)sizeof(bf16_t);  // keys (and values) of a step
constexpr float kSumLimit = 65536.f;      // of 16 exponentials, beyond which the maximum is looked at
constexpr float kLazy = 8.f;              // and followed where it has grown by 2^8

// 16 bytes per lane straight to LDS: lane l's land 16 l bytes behind the wavefront's `dst`.  From a base that is the same
// for the wavefront and 32 bits of offset a lane; to_lds_far from any address.  (After loads of the second kind the compiler
// takes every wait for LDS to be a wait for all of LDS, as it does for accesses through generic pointers.)
// STREAM: past the caches.
template <bool STREAM>
__device__ __forceinline__ void to_lds(const void* base, uint32_t bytes, uint32_t off, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000),
                                           (__attribute__((address_space(3))) void*)dst, 16, (int)off, 0, 0, STREAM ? 2 : 0);
#endif
}
__device__ __forceinline__ void to_lds_far(const void* src, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
#endif
}

// A 4 x 16 block of bf16 by columns: of the 16 lanes of a row, lane i names four neighbours, piece i % 4 of block row i / 4,
// and gets column i of the block.
__device__ __forceinline__ u32x2 lds_columns(const unsigned char* at) {
#ifdef __HIP_DEVICE_COMPILE__
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
  return __builtin_bit_cast(u32x2, v);
#else
  return (u32x2){0u, 0u};
#endif
}

// Largest of 16 products times `c`, over both halves of the wavefront.  (v_max3 without the canonicalisation that fmaxf
// brings along.  In front of assembly the compiler leaves no time for products to reach their registers; it does in front
// of the multiplication, and the empty assembly puts the rest behind it.)
__device__ __forceinline__ float top16(f32x16& s, float c) {
  const auto max3 = [](float x, float y, float z) {
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(x), "v"(y), "v"(z));
    return d;
  };
  const float last = s[15] * c;
  asm volatile("" : "+v"(s) : "v"(last));
  const float a = max3(s[0], s[1], s[2]), b = max3(s[3], s[4], s[5]), d = max3(s[6], s[7], s[8]);
  const float e = max3(s[9], s[10], s[11]), f = max3(s[12], s[13], s[14]);
  const float mine = fmaxf(max3(max3(a, b, d), e, f) * c, last);
  const SwapPair sw = swap_rows32(__float_as_uint(mine));
  return fmaxf(__uint_as_float(sw.a), __uint_as_float(sw.b));
}

// `sum` and two weights as they are after rounding
__device__ __forceinline__ float add_rounded(uint32_t pair, float sum) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
#else
  return sum;
#endif
}

}  // namespace

struct ChunkAttendArgs {
  ChunkView ch;
  const bf16_t* q;
  bf16_t* out;
  float* out_lse;
  float* partial;     // [workgroup][rows][128] sums of the parts; null: no tile is ever cut
  float2* part_stats; // [workgroup][rows] their maxima and sums of exponentials
  int4* part_place;   // [workgroup] what the merge needs: first row in the packed tensors, rows and part, parts, ChunkPlace::next
  int tile_tokens;    // tokens of a row tile
  int slots, most;    // workgroups the chip holds at a time; parts at most
};

// Where a workgroup works: tile `tile` of sequence b, part `part` of `parts` of its keys.
struct ChunkPlace {
  int b, tile, part, parts;
  int first, next;  // indexes among all parts of a KV head: of the tile's first part, and how much further each other is
};

struct ChunkSeq {
  int row, n, len;  // first row and rows in the packed tensors, tokens in the cache (the new ones among them)
};
__device__ __forceinline__ ChunkSeq chunk_seq(const CacheView& c, const ChunkView& ch, int b) {
  ChunkSeq s;
  s.row = chunk_first(ch, b);
  s.n = chunk_rows(ch, b);
  const int cap = c.pages_cap * c.page_size, n = c.seq_lens[b];
  s.len = n < 0 ? 0 : (n > cap ? cap : n);
  return s;
}

// Every wavefront derives the same division from the lengths.  `own`: sequence `lane` of the first 64, which most batches
// are all of: looked up once, as each look is a round trip that nothing hides.
__device__ __forceinline__ ChunkSeq chunk_seq_of_lane(const CacheView& c, const ChunkView& ch) {
  const int lane = threadIdx.x % kWave;
  if (lane < c.batch) return chunk_seq(c, ch, lane);
  return {0, 0, 0};
}
__device__ __forceinline__ int chunk_size_for(const CacheView& c, const ChunkAttendArgs& a, const ChunkSeq& own) {
  const int lane = threadIdx.x % kWave;
  if (!a.partial) return kChunkWhole;
  const auto total = [](int x) { return __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)x), kWave - 1); };
  ChunkLoad load = {0, 0.f, 0};
  const auto each = [&](const auto& fn) {  // of the tiles and steps of every sequence
    for (int b0 = 0; b0 < c.batch; b0 += kWave) {
      int t = 0, steps = 0;
      if (b0 + lane < c.batch) {
        const ChunkSeq s = b0 == 0 ? own : chunk_seq(c, a.ch, b0 + lane);
        t = chunk_ceil(s.n, a.tile_tokens);
        steps = t ? chunk_ceil(s.len, kStep) : 0;
      }
      fn(t, steps);
    }
  };
  each([&](int t, int steps) {
    load.tiles += total(t) * c.n_kv_heads;
    // (a coarser count keeps the sums in range where sequences are long: 2^15 steps are 2^21 tokens)
    load.work += (float)total(min(t, a.most) * min(steps, 1 << 15)) * (float)c.n_kv_heads;
    load.longest = max(load.longest, (int)wave_max_u32((uint32_t)steps));
  });
  return chunk_part_size(load, a.slots, a.most, [&](int size) {
    int n = 0;
    each([&](int t, int steps) { n += total(t * chunk_parts(steps, size)); });
    return n * c.n_kv_heads;
  });
}

__device__ __forceinline__ bool chunk_place(const CacheView& c, const ChunkAttendArgs& a, const ChunkSeq& own, int size, int at,
                                            ChunkPlace& p, ChunkSeq& s) {
  int idx;
  if (!locate_tile(c.batch, at, [&](int i) {
        const ChunkSeq s = i < kWave ? own : chunk_seq(c, a.ch, i);
        return chunk_ceil(s.n, a.tile_tokens) * chunk_parts(chunk_ceil(s.len, kStep), size);
      }, p.b, idx))
    return false;
  if (p.b < kWave) s = {__builtin_amdgcn_readlane(own.row, p.b), __builtin_amdgcn_readlane(own.n, p.b), __builtin_amdgcn_readlane(own.len, p.b)};
  else s = chunk_seq(c, a.ch, p.b);
  p.parts = chunk_parts(chunk_ceil(s.len, kStep), size);
  // the tiles of one part side by side, as they read the same keys; those that see most first
  p.next = chunk_ceil(s.n, a.tile_tokens);
  p.part = idx / p.next;
  p.tile = p.next - 1 - idx % p.next;
  p.first = at - p.part * p.next;
  return true;
}

template <bool TOK, bool FAR, int WAVES, bool STREAM>
__global__ __launch_bounds__(WAVES * kWave) __attribute__((amdgpu_waves_per_eu(2)))
void chunk_attend_kernel(CacheView c, ChunkAttendArgs a) {
  constexpr int kWaveTok = kStep / WAVES;  // tokens a wavefront brings
  extern __shared__ __align__(256) unsigned char s_tiles[];          // [2] keys, [2] values
  constexpr int kRows = WAVES * 32;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, h = lane / 32;
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads;
  ChunkPlace pl;
  ChunkSeq s;
  const ChunkSeq own = chunk_seq_of_lane(c, a.ch);
  const bool any = chunk_place(c, a, own, chunk_size_for(c, a, own), at, pl, s);
  const bool holds = a.partial && (int)blockIdx.x < a.most;  // a place for a part's rows
  if (!any) {
    if (holds && threadIdx.x == 0) a.part_place[blockIdx.x] = make_int4(0, 0, 1, 0);
    return;
  }
  if (pl.parts > 1 && !holds) return;  // (`starts` that overlap)
  const int G = c.group, ps = c.page_size;
  const int t0 = pl.tile * a.tile_tokens, nt = min(a.tile_tokens, s.n - t0);
  const int rows = nt * G;
  if (holds && threadIdx.x == 0) a.part_place[blockIdx.x] = make_int4(s.row + t0, rows << 16 | pl.part, pl.parts, pl.next);
  const int pos0 = s.len - s.n + t0;  // place in the cache of the tile's first token

  // the part's steps
  const int steps = chunk_ceil(max(0, min(s.len, pos0 + nt)), kStep), per = chunk_ceil(steps, pl.parts);
  const int it0 = min(pl.part * per, steps), it1 = min(it0 + per, steps);

  // this lane's row: its query in registers, and the last key it sees
  const int r = wave * 32 + col;
  const bool working = wave * 32 < rows;
  const int last = r < rows ? pos0 + r / G : -1;
  const auto packed_row = [&](int r) {  // (token, head) of the packed tensors
    const int t = r / G;
    return (int64_t)(s.row + t0 + t) * c.n_q_heads + (int64_t)g * G + (r - t * G);
  };
  bf16x8 qf[8];
  {
    const bf16_t* qp = a.q + packed_row(min(r, rows - 1)) * kHeadDim + h * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 v = *reinterpret_cast<const u32x4*>(qp + j * 16);
      if (r >= rows) v = (u32x4){0u, 0u, 0u, 0u};
      qf[j] = as_bf16x8(v);
    }
  }
  const int sees_first = working ? pos0 + wave * 32 / G : -1;  // the last key that all of the wavefront's rows see

  // Keys and values of a step to LDS: every wavefront brings kWaveTok tokens of each, 16 bytes a lane.
  //   keys: [64][16 chunks], chunk x of row r at x ^ r % 16, so that 32 rows at one chunk spread over the banks
  //   values by channel: per page [8 blocks of 16 channels][2 halves of its tokens][16 channels], so that 16 lanes read 256
  //   bytes in a row; by token: [64][16 chunks], chunk x of row r at x ^ 4 (r % 4)
  constexpr int kLoads = kWaveTok / 4;        // of keys, and of values, a wavefront issues for a step: 1 KiB each
  typedef typename std::conditional<TOK && !FAR, uint32_t, int64_t>::type Offset;  // bytes from the pool's beginning
  const int first_tok = wave * kWaveTok;      // of the step
  const int64_t head_off = (int64_t)g * c.stride_head * sizeof(bf16_t), page_off = c.stride_page * sizeof(bf16_t);
  // Looked up a step ahead, by every wavefront for the whole step: lane i token i of it, or page i where pages are tiles.
  int page = 0, slot = 0, raw = -1;
  Offset off_k = 0, off_v = 0;  // where the step's rows lie: of the keys to be requested, of the values
  const auto in_range = [&](int raw) { return raw >= 0 && (int64_t)raw < c.n_phys_pages; };
  const auto look_up = [&](int it) {
    const int t0 = it * kStep, end = it < it1 ? s.len : 0;
    if (TOK) raw = t0 + lane < end ? phys_page_request(c, pl.b, page) : -1;
    else raw = lane < kStep / kAttnPage && t0 + lane * kAttnPage < end ? phys_page_request(c, pl.b, t0 / kAttnPage + lane) : -1;
  };
  if (TOK) {
    page = (it0 * kStep + lane) / ps;
    slot = it0 * kStep + lane - page * ps;
  }
  const int skip_pages = kStep / ps, skip_slots = kStep - skip_pages * ps;
  // 16 bytes a lane from the row of token `r` of the step, whose offset is with lane r
  const auto row_to_lds = [&](const bf16_t* pool, Offset off, int r, int from, unsigned char* dst) {
    const uint32_t lo = (uint32_t)__shfl((int)off, r);
    if (FAR) {
      const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)((int64_t)off >> 32), r) << 32 | lo);
      to_lds_far(reinterpret_cast<const char*>(pool) + at + from, dst);
    } else {
      to_lds<STREAM>(pool, 0xffffffffu, lo + from, dst);
    }
  };
  // Keys of step `it`, looked up before; looks up the next one.  Returns a bit per token of the step that exists.
  const auto issue_keys = [&](int it, auto to) {
    unsigned char* kb = s_tiles + decltype(to)::value * kKeyBytes + first_tok * 256;
    unsigned long long valid = __ballot(in_range(raw));
    if (TOK) {
      off_k = in_range(raw) ? (Offset)(raw * page_off + head_off + slot * (kHeadDim * (int)sizeof(bf16_t))) : (Offset)0;
      slot += skip_slots;
      page += skip_pages;
      if (slot >= ps) { slot -= ps; ++page; }
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {  // 16 lanes a row
        const int r = first_tok + 4 * j + lane / 16;
        row_to_lds(c.k_pool, off_k, r, ((lane % 16) ^ r % 16) * 16, kb + j * 1024);
      }
    } else {
      const int mine = __builtin_amdgcn_readlane(raw, first_tok / kAttnPage);
      off_k = in_range(mine) ? (Offset)(mine * page_off + head_off) : (Offset)0;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int r = first_tok % kAttnPage + 4 * j + lane / 16;
        to_lds<STREAM>(reinterpret_cast<const char*>(c.k_pool) + off_k, 4096, r * 256 + ((lane % 16) ^ r) * 16, kb + j * 1024);
      }
      const int left = s.len - it * kStep;
      if (valid == 0xfull && left >= kStep) {
        valid = ~0ull;
      } else {
        unsigned long long tokens = 0;
#pragma unroll
        for (int x = 0; x < kStep / kAttnPage; ++x) tokens |= (valid >> x & 1ull) * 0xffffull << 16 * x;
        valid = left >= kStep ? tokens : left > 0 ? tokens & ((1ull << left) - 1ull) : 0ull;
      }
    }
    look_up(it + 1);
    return valid;
  };
  const auto issue_values = [&](auto to) {  // of the step whose offsets are in off_v
    unsigned char* vb = s_tiles + (2 + decltype(to)::value) * kKeyBytes + first_tok * 256;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      if (TOK) {
        const int r = first_tok + 4 * j + lane / 16;
        row_to_lds(c.v_pool, off_v, r, ((lane % 16) ^ 4 * (lane / 16)) * 16, vb + j * 1024);
      } else {
        to_lds<STREAM>(reinterpret_cast<const char*>(c.v_pool) + off_v, 4096,
               (first_tok % kAttnPage / 4 + j) * 1024 + lane / 32 * 512 + lane % 16 * 32 + lane / 16 % 2 * 16, vb + j * 1024);
      }
    }
  };

  f32x16 O[4];
  float m = kNegBig, l = 0.f, lr = 0.f;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) O[cb] = f32x16{};
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  // token of the tile whose keys this lane reads as row `col` of a product: bits 2 and 3 swapped
  const int key_row = (col & 0x13) | (col & 4) << 1 | (col & 8) >> 1;

  // Chunk 2 j + h of this lane's row stands at (2 j + h) ^ key_row % 16.  `at`: key_at, kept from being turned into eight
  // registers outside the loop.
  const uint32_t key_at = (uint32_t)(key_row * 256 + (h ^ (key_row & 15)) * 16);
  const auto read_key = [&](uint32_t at, auto slot, int u, int j, bf16x8& kf) {
    kf = as_bf16x8(*reinterpret_cast<const u32x4*>(s_tiles + (at ^ (uint32_t)(32 * j)) + (decltype(slot)::value * kKeyBytes + u * 8192)));
  };
  // Channels 32 cb + col, tokens 32 u + 16 y + 8 h + 0..7.  By token, lane i of a row of 16 names a piece of token row
  // 4 z + i / 4 (z: first or second four) and of 16 channels; 32 lanes, four token rows, read one after the other, and their
  // chunks 4 cb + 0..3 stand at 4 (cb ^ i / 4) + 0..3, a place of its own for each.
  const int vi = lane % 16;
  const uint32_t value_at = TOK ? (uint32_t)((8 * h + vi / 4) * 256 + vi % 2 * 8 + (4 * (vi / 4) + 2 * (lane / 16 % 2) + vi % 4 / 2) * 16)
                                : (uint32_t)(col / 16 * 512 + h * 256 + col % 16 * 16);
  const auto read_value = [&](uint32_t at, auto slot, int u, int y, int cb, u32x4& vf) {
    const int base = (2 + decltype(slot)::value) * kKeyBytes + u * 8192;
    if (TOK) {
      u32x2 w[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) w[z] = lds_columns(s_tiles + (at ^ (uint32_t)(64 * cb)) + (base + (16 * y + 4 * z) * 256));
      vf = (u32x4){w[0].x, w[0].y, w[1].x, w[1].y};
    } else {
      vf = *reinterpret_cast<const u32x4*>(s_tiles + value_at + (base + y * 4096 + cb * 1024));
    }
  };
  const auto mask = [&](f32x16& S, int key0, uint32_t ok) {
    const uint32_t there = ok >> (8 * h);
    const int seen = last - key0 - 8 * h;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int t = 16 * (i / 8) + i % 8;
      if (!((there >> t) & 1u) || t > seen) S[i] = -INFINITY;
    }
  };
  // exp2 of the logits relative to m, rounded for the second product, and their sum.  The running maximum is not followed
  // key by key: a sum that stays below 2^16 has lost nothing to being formed relative to an older maximum.  Only where one
  // does not (the first keys of a row, relative to kNegBig, always), the maximum of these logits is taken, sums so far are
  // scaled to it where it exceeds the old one by 2^8, and the exponentials are formed again.
  const auto exponential = [&](float x) { return fast_exp2(fmaf(x, sc, -m)); };
  const auto follow_maximum = [&](f32x16& S, float& sum, u32x4 (&pf)[2]) {
    const float mx = top16(S, sc);
    const bool up = mx > m + kLazy;
    const float mn = up ? mx : m, alpha = fast_exp2(m - mn);
    m = mn;
    l *= alpha;
    lr *= alpha;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) O[cb] *= alpha;
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = exponential(S[2 * j]), y = exponential(S[2 * j + 1]);
      sum += x + y;
      pf[j / 4][j % 4] = pack_bf16x2(x, y);
    }
  };
  // What lies where no token is may be anything, and 0 x NaN is not 0: the wavefront that brought such values clears them
  // once they are there.
  const auto clear_values = [&](auto slot, unsigned long long valid) {
    if (valid == ~0ull) return;
    unsigned char* vb = s_tiles + (2 + decltype(slot)::value) * kKeyBytes + first_tok * 256;
    const uint32_t live = (uint32_t)(valid >> (TOK ? first_tok : first_tok / kAttnPage * kAttnPage));
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      u32x4* at = reinterpret_cast<u32x4*>(vb + j * 1024 + lane * 16);
      if (TOK) {
        if (!((live >> (4 * j + lane / 16)) & 1u)) *at = (u32x4){0u, 0u, 0u, 0u};
      } else {  // eight tokens of a channel
        const uint32_t bits = live >> (8 * (lane / 16 % 2));
        u32x4 v = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] &= (((bits >> (2 * e)) & 1u) ? 0x0000ffffu : 0u) | (((bits >> (2 * e + 1)) & 1u) ? 0xffff0000u : 0u);
        *at = v;
      }
    }
  };

  // A value that is not finite belongs to the rows that see its key, and 0 x NaN would carry it to the others of the tile.
  // Where there are such values among partly seen keys, the unit's keys with any are added one by one, for the rows that
  // see them, and leave the operand.
  const auto keep_future_out = [&](int key0, u32x4 (&vf)[2][4], u32x4 (&pf)[2]) {
    uint32_t odd = 0;  // bit 8 y + e: key 16 y + 8 h + e has one among this lane's channels
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          odd |= (vf[y][cb][i] & 0x7f80u) == 0x7f80u ? 1u << (8 * y + 2 * i) : 0u;
          odd |= (vf[y][cb][i] & 0x7f800000u) == 0x7f800000u ? 2u << (8 * y + 2 * i) : 0u;
        }
    if (!__any(odd != 0u)) return;
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll 1
      for (int k = 0; k < 16; ++k) {  // key 16 y + k, element k % 8 of the lanes of half k / 8
        if (!__any(h == k / 8 && (odd >> (8 * y + k % 8) & 1u))) continue;
        const uint32_t mine = h == k / 8 ? k & 1 ? 0xffff0000u : 0xffffu : 0u;
        const u32x4 sel = {k % 8 / 2 == 0 ? mine : 0u, k % 8 / 2 == 1 ? mine : 0u, k % 8 / 2 == 2 ? mine : 0u, k % 8 / 2 == 3 ? mine : 0u};
        const bool seen = key0 + 16 * y + k <= last;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          const f32x16 sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[y][cb] & sel), as_bf16x8(pf[y] & sel), O[cb], 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) O[cb][i] = seen ? sum[i] : O[cb][i];
          vf[y][cb] &= ~sel;
        }
      }
  };
  const auto partly = [&](int it, unsigned long long valid) { return valid != ~0ull || it * kStep + kStep - 1 > sees_first; };
  // A unit is 32 keys.  Its exponentials (S holds its logits) stand beside the next unit's products, a matrix instruction
  // and what fits under it at a time; then its values are added while the keys of the unit after the next come in.  So
  // in step `it` the values of `it` are read and the keys of it + 1.
  bf16x8 kf[8];
  f32x16 S;
  unsigned long long valid0 = 0, valid1 = 0;  // tokens that exist: of the step, and of the next one
  const auto fence = []() { __builtin_amdgcn_sched_barrier(0); };
  const auto step = [&](int it, auto slot) {
    constexpr std::integral_constant<int, 1 - decltype(slot)::value> other{};
    __builtin_amdgcn_s_waitcnt(0);  // this wavefront's share has landed
    clear_values(slot, valid0);
    __syncthreads();                // everyone's has, and what the last step used is free
    off_v = off_k;
    issue_values(other);  // (behind the last step: from the pools' beginning, and unused)
    const unsigned long long valid2 = issue_keys(it + 2, slot);
    const bool masked0 = partly(it, valid0), masked1 = it + 1 < it1 && partly(it + 1, valid1);
    const unsigned long long seen0 = valid0, seen1 = valid1;
    valid0 = valid1;
    valid1 = valid2;
    if (!working) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x16 N;
      const uint32_t keys = use_late(key_at);
      u32x4 vf[2][4], pf[2];
      float sums[8];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        fence();
        N = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[j], j == 0 ? f32x16{} : N, 0, 0, 0);
        read_value(value_at, slot, u, j / 4, j % 4, vf[j / 4][j % 4]);
        const float x = exponential(S[2 * j]), y = exponential(S[2 * j + 1]);
        sums[j] = x + y;
        pf[j / 4][j % 4] = pack_bf16x2(x, y);
      }
      fence();
      __builtin_amdgcn_s_setprio(0);
      float sum = ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
      float rounded = sum;
      if (__any(!(sum <= fminf(kSumLimit, l)))) {
        if (__any(!(sum <= kSumLimit))) follow_maximum(S, sum, pf);
        rounded = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) rounded = add_rounded(pf[j / 4][j % 4], rounded);
      }
      l += sum;
      lr += rounded;
      if (masked0) keep_future_out(it * kStep + 32 * u, vf, pf);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        fence();
        O[j % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf[j / 4][j % 4]), as_bf16x8(pf[j / 4]), O[j % 4], 0, 0, 0);
        read_key(keys, other, u, j, kf[j]);  // (behind the last step: of keys that are not there, and go unused)
      }
      fence();
      S = N;
      if (u == 0 ? masked0 : masked1) mask(S, it * kStep + 32 * (u + 1), (uint32_t)(u == 0 ? seen0 >> 32 : seen1));
    }
  };
  if (it0 < it1) {
    look_up(it0);
    valid0 = issue_keys(it0, std::integral_constant<int, 0>{});
    off_v = off_k;
    issue_values(std::integral_constant<int, 0>{});
    valid1 = issue_keys(it0 + 1, std::integral_constant<int, 1>{});
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (working) {  // the first unit's logits, and the keys of the second
      constexpr std::integral_constant<int, 0> slot{};
#pragma unroll
      for (int j = 0; j < 8; ++j) read_key(key_at, slot, 0, j, kf[j]);
#pragma unroll
      for (int j = 0; j < 8; ++j) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j], qf[j], j == 0 ? f32x16{} : S, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) read_key(key_at, slot, 1, j, kf[j]);
      if (partly(it0, valid0)) mask(S, it0 * kStep, (uint32_t)valid0);
    }
  }
  for (int it = it0; it < it1; it += 2) {
    step(it, std::integral_constant<int, 0>{});
    if (it + 1 < it1) step(it + 1, std::integral_constant<int, 1>{});
  }

  const auto both_halves = [](float x) {
    const SwapPair sw = swap_rows32(__float_as_uint(x));
    return __uint_as_float(sw.a) + __uint_as_float(sw.b);
  };
  const float sum = both_halves(l), rounded = both_halves(lr);
  if (r >= rows) return;
  if (pl.parts > 1) {
    const int64_t at_row = ((int64_t)at * c.n_kv_heads + g) * kRows + r;
    float* part = a.partial + at_row * kHeadDim;
    const float fit = sum == 0.f ? 0.f : sum / rounded;  // (so that the merge needs one sum)
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(part + 32 * cb + 2 * i + 4 * h) = make_float4(O[cb][i] * fit, O[cb][i + 1] * fit, O[cb][i + 2] * fit, O[cb][i + 3] * fit);
    if (h == 0) a.part_stats[at_row] = make_float2(m, sum);
    return;
  }
  const int64_t row = packed_row((int)use_late((uint32_t)r));
  const float inv = sum == 0.f ? 0.f : 1.f / rounded;  // (a sum that is NaN stays one, here and below: only 0 is no key at all)
  bf16_t* o = a.out + row * kHeadDim + 4 * h;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<u32x2*>(o + 32 * cb + 2 * i) =
          (u32x2){pack_bf16x2(O[cb][i] * inv, O[cb][i + 1] * inv), pack_bf16x2(O[cb][i + 2] * inv, O[cb][i + 3] * inv)};
  if (a.out_lse && h == 0) a.out_lse[row] = sum == 0.f ? -INFINITY : (m + __log2f(sum)) * kLn2;
}

constexpr int kMergeWaves = 8, kMergeSlices = 2;  // wavefronts to a workgroup, workgroups to a part

// The parts of a tile joined: a wavefront per row, a lane per two channels.  A row is a chain of dependent reads, so it is
// wavefronts at work that count: 16 per part were 2 to 35 % of a whole call better than 4.
__global__ __launch_bounds__(kMergeWaves * kWave) void chunk_merge_kernel(CacheView c, ChunkAttendArgs a, int tile_rows) {
  const int4 place = a.part_place[blockIdx.x];
  const int parts = place.z;
  if (parts == 1) return;
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads, G = c.group;
  const int rows = place.y >> 16, part = place.y & 0xffff, first = at - part * place.w;
  const int lane = threadIdx.x % kWave;
  const int64_t next = (int64_t)place.w * c.n_kv_heads * tile_rows;  // rows from part to part
  // the tile's parts share its rows
  for (int r = part + parts * (threadIdx.x / kWave + kMergeWaves * blockIdx.y); r < rows; r += parts * kMergeWaves * kMergeSlices) {
    const int64_t row0 = ((int64_t)first * c.n_kv_heads + g) * tile_rows + r;
    const float* p = a.partial + row0 * kHeadDim;
    const float2* stats = a.part_stats + row0;
    float m = kNegBig;
    for (int i = lane; i < parts; i += kWave) m = fmaxf(m, stats[i * next].x);
    m = wave_max_f32(m);
    float l = 0.f, x = 0.f, y = 0.f;
    for (int i0 = 0; i0 < parts; i0 += kWave) {
      const int n = min(kWave, parts - i0);
      float w = 0.f;
      if (lane < n) {
        const float2 ml = stats[(i0 + lane) * next];
        w = fast_exp2(ml.x - m);
        l = fmaf(ml.y, w, l);
      }
      const float* o = p + i0 * next * kHeadDim + 2 * lane;
      for (int i = 0; i < n; i += 4) {  // (absent ones weigh nothing, and read the last)
        float2 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float2*>(o + min(i + u, n - 1) * next * kHeadDim);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float wu = i + u < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), (i + u) % kWave)) : 0.f;
          x = fmaf(v[u].x, wu, x);
          y = fmaf(v[u].y, wu, y);
        }
      }
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) l += __shfl_xor(l, d);
    const int t = r / G;
    const int64_t row = (int64_t)(place.x + t) * c.n_q_heads + (int64_t)g * G + r - t * G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint32_t*>(a.out + row * kHeadDim + 2 * lane) = pack_bf16x2(x * inv, y * inv);
    if (a.out_lse && lane == 0) a.out_lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
  }
}

ChunkPlan plan_chunk_attend(const CacheView& c, int n_tokens) {
  ChunkPlan p;
  // 32 bits reach every row of a token-major pool whose last tile ends below 4 GiB
  const int64_t end = (c.n_phys_pages - 1) * c.stride_page + (c.n_kv_heads - 1) * c.stride_head + (int64_t)c.page_size * kHeadDim;
  p.far = c.v_token_major && end * (int64_t)sizeof(bf16_t) >= (int64_t)1 << 32;
  const int64_t held = (int64_t)c.batch * c.pages_cap * c.page_size * c.n_kv_heads * kHeadDim * 2 * (int64_t)sizeof(bf16_t);
  const int64_t rows = (int64_t)n_tokens * c.group / c.batch;  // of a sequence on average
  p.tile_rows = chunk_tile_rows(p.far, rows, held);
  p.tile_tokens = p.tile_rows / c.group;
  p.stream = chunk_past_caches(p.far, rows, held);
  p.slots = 256 * (256 / p.tile_rows);
  const int64_t at_least = ((int64_t)n_tokens + p.tile_tokens - 1) / p.tile_tokens * c.n_kv_heads;
  int64_t tiles = (int64_t)n_tokens / p.tile_tokens + c.batch;
  if (tiles > n_tokens) tiles = n_tokens;
  tiles *= c.n_kv_heads;
  const int rounds = chunk_rounds(at_least, p.slots);
  p.most = p.slots * rounds;
  // Where no sequence can be long enough to be cut, neither the merge nor the workgroups of parts are launched: a prompt of
  // 300 tokens 14.9 us, 17.2 with them.
  p.cuts = at_least < p.most && (int64_t)c.pages_cap * c.page_size > kChunkShort * kStep;
  p.workgroups = p.cuts && tiles < p.most ? p.most : tiles;
  // (for any number of tokens, so that what serves many serves few)
  p.total_bytes = n_tokens ? (size_t)ROCKETKV_WS_HEADER_BYTES + (size_t)256 * kChunkRounds * (256 * (kHeadDim + 2) * sizeof(float) + 2 * sizeof(int4)) : 0;
  return p;
}

hipError_t launch_chunk_attend(const CacheView& c, const ChunkView& ch, const bf16_t* q, bf16_t* out, float* out_lse,
                               void* ws, const ChunkPlan& plan, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  ChunkAttendArgs a;
  a.ch = ch;
  a.q = q;
  a.out = out;
  a.out_lse = out_lse;
  const int64_t part_rows = (int64_t)plan.most * plan.tile_rows;
  a.partial = plan.cuts ? reinterpret_cast<float*>(static_cast<char*>(ws) + ROCKETKV_WS_HEADER_BYTES) : nullptr;
  a.part_stats = plan.cuts ? reinterpret_cast<float2*>(a.partial + part_rows * kHeadDim) : nullptr;
  a.part_place = plan.cuts ? reinterpret_cast<int4*>(a.part_stats + part_rows) : nullptr;
  a.tile_tokens = plan.tile_tokens;
  a.slots = plan.slots;
  a.most = plan.most;
  const auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.workgroups), dim3(waves * kWave), 4 * kKeyBytes, st, c, a);
  };
  if (plan.far) launch(chunk_attend_kernel<true, true, 8, false>, 8);
  else if (plan.tile_rows == 256 && c.v_token_major) launch(chunk_attend_kernel<true, false, 8, false>, 8);
  else if (plan.tile_rows == 256) launch(chunk_attend_kernel<false, false, 8, false>, 8);
  else if (c.v_token_major && plan.stream) launch(chunk_attend_kernel<true, false, 4, true>, 4);
  else if (c.v_token_major) launch(chunk_attend_kernel<true, false, 4, false>, 4);
  else if (plan.stream) launch(chunk_attend_kernel<false, false, 4, true>, 4);
  else launch(chunk_attend_kernel<false, false, 4, false>, 4);
  if (plan.cuts) {
    hipLaunchKernelGGL(chunk_merge_kernel, dim3(plan.most, kMergeSlices), dim3(kMergeWaves * kWave), 0, st, c, a, plan.tile_rows);
  }
  return hipGetLastError();
}

}  // namespace rkv
