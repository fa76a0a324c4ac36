// Causal attention of a chunk of new tokens over the paged cache they have been put into: whole prompts, the next piece
// of a prompt, a turn, drafted tokens, single tokens, in any mixture.
//
// Rows of a (sequence, KV head) are its new tokens times the group's query heads, so every key serves the whole group.
// A workgroup takes a tile of rows, 32 or 64 to a wavefront, and walks the keys 64 at a time through LDS, one pass with
// the running maximum m and sum l of each row:
//
//   S^T[key][row]     = K[key][:] . Q[row][:]              A = keys (32 rows), B = queries, kept in registers
//   O^T[chan][row]   += V^T[chan][key] . P^T[key][row]     A = values by channel, B = exp2(S c - m)
//
// Both products have the row as their column, so a lane owns one row: its 16 logits of a product, maximum, sum and
// outputs never leave it, but for one exchange with the lane 32 further, which holds the same row's other keys.  The
// product leaves a lane the keys of A's rows 8a + 4h + r; with the rows of K read in an order that swaps bits 2 and 3,
// these are keys 16x + 8h + 0..7, which packed to bf16 are the second product's operand as they stand.  P is rounded to
// bf16 there (relative 2^-9 at most each, the sum l takes the unrounded values); everything else is fp32.
#include "attend_core.h"
#include "chunk_division.h"

namespace rkv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;                                        // keys per step
constexpr int kKeyBytes = kStep * kHeadDim * (int)sizeof(bf16_t);  // keys (and values) of a step
constexpr int kChunkT = 256;
constexpr int kRowStride = kHeadDim + 2;  // a row of a part: O[128], maximum, sum
constexpr float kLazy = 8.f;              // a maximum may be exceeded by a factor of 2^8 before sums are scaled anew

// 16 bytes per lane from `src` straight to LDS: lane l's land 16 l bytes behind the wavefront's `dst`
__device__ __forceinline__ void to_lds(const bf16_t* src, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
#endif
}

// Four bf16 of a column each: the 16 lanes of a row name 16 pieces of four neighbours, four rows of four pieces; lane i
// gets element i % 4 + 4 ... of the transposed block: column i of the 16, rows 0..3.
__device__ __forceinline__ u32x2 lds_columns(const unsigned char* at) {
#ifdef __HIP_DEVICE_COMPILE__
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
  return __builtin_bit_cast(u32x2, v);
#else
  return (u32x2){0u, 0u};
#endif
}

}  // namespace

struct ChunkAttendArgs {
  ChunkView ch;
  const bf16_t* q;
  bf16_t* out;
  float* out_lse;
  float* partial;     // [workgroup][rows][kRowStride]; null: no tile is ever cut
  int tile_tokens;    // tokens of a row tile
  int target;         // workgroups wanted where there are fewer tiles
};

// Where a workgroup works: tile `tile` of sequence b, part `part` of `parts` of its keys.
struct ChunkPlace {
  int b, tile, part, parts;
  int first;  // index of the tile's first part among all parts of a KV head
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

// Every wavefront derives the same division from the lengths.
__device__ __forceinline__ int chunk_size_for(const CacheView& c, const ChunkAttendArgs& a) {
  const int lane = threadIdx.x % kWave;
  if (!a.partial) return kChunkWhole;
  int64_t work = 0, tiles = 0;
  int longest = 0;
  const auto total = [](int x) { return __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)x), kWave - 1); };
  for (int b0 = 0; b0 < c.batch; b0 += kWave) {
    int t = 0, steps = 0;
    if (b0 + lane < c.batch) {
      const ChunkSeq s = chunk_seq(c, a.ch, b0 + lane);
      t = chunk_ceil(s.n, a.tile_tokens);
      steps = t ? chunk_ceil(s.len, kStep) : 0;
    }
    tiles += total(t);
    // (tiles are fewer than `target` where this counts, so that products of the sums stay far below 2^31)
    work += (int64_t)total(min(t, a.target) * min(steps, (1 << 30) / a.target / kWave));
    longest = max(longest, (int)wave_max_u32((uint32_t)steps));
  }
  return chunk_part_size(tiles * c.n_kv_heads, work * c.n_kv_heads, a.target, longest, [&](int size) {
    int64_t n = 0;
    for (int b0 = 0; b0 < c.batch; b0 += kWave) {
      int x = 0;
      if (b0 + lane < c.batch) {
        const ChunkSeq s = chunk_seq(c, a.ch, b0 + lane);
        x = chunk_ceil(s.n, a.tile_tokens) * chunk_parts(chunk_ceil(s.len, kStep), size);
      }
      n += total(x);
    }
    return n * c.n_kv_heads;
  });
}

__device__ __forceinline__ bool chunk_place(const CacheView& c, const ChunkAttendArgs& a, int size, int at, ChunkPlace& p) {
  int idx;
  if (!locate_tile(c.batch, at, [&](int i) {
        const ChunkSeq s = chunk_seq(c, a.ch, i);
        return chunk_ceil(s.n, a.tile_tokens) * chunk_parts(chunk_ceil(s.len, kStep), size);
      }, p.b, idx))
    return false;
  const ChunkSeq s = chunk_seq(c, a.ch, p.b);
  p.parts = chunk_parts(chunk_ceil(s.len, kStep), size);
  const int tiles = chunk_ceil(s.n, a.tile_tokens);
  p.part = idx % p.parts;
  p.first = at - p.part;
  p.tile = tiles - 1 - idx / p.parts;  // the tiles that see most come first
  return true;
}

template <bool TOK, int NB>
__global__ __launch_bounds__(kChunkT) __attribute__((amdgpu_waves_per_eu(NB == 1 ? 2 : 1)))
void chunk_attend_kernel(CacheView c, ChunkAttendArgs a) {
  extern __shared__ __align__(16) unsigned char s_tiles[];  // [2][keys, values]
  __shared__ __align__(8) uint16_t s_valid[2][kStep / 16];  // the step's tokens that exist
  constexpr int kRows = 4 * 32 * NB;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, h = lane / 32;
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads;
  ChunkPlace pl;
  if (!chunk_place(c, a, chunk_size_for(c, a), at, pl)) return;
  if (pl.parts > 1 && (int)blockIdx.x >= a.target) return;  // (`starts` that overlap: no place for its rows)
  const ChunkSeq s = chunk_seq(c, a.ch, pl.b);
  const int G = c.group, ps = c.page_size;
  const int t0 = pl.tile * a.tile_tokens, nt = min(a.tile_tokens, s.n - t0);
  const int rows = nt * G;
  const int64_t lane_row0 = s.row + t0;
  const int pos0 = s.len - s.n + t0;  // place in the cache of the tile's first token

  // the part's steps
  const int steps = chunk_ceil(max(0, min(s.len, pos0 + nt)), kStep), per = chunk_ceil(steps, pl.parts);
  const int it0 = min(pl.part * per, steps), it1 = min(it0 + per, steps);

  // this wavefront's rows: queries in registers, and the last key each row sees
  bf16x8 qf[NB][8];
  int last[NB], tok[NB], head[NB];
  bool real[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const int r = (wave * NB + x) * 32 + col;
    real[x] = r < rows;
    tok[x] = real[x] ? r / G : 0;
    head[x] = real[x] ? r - tok[x] * G : 0;
    last[x] = real[x] ? pos0 + tok[x] : -1;
    const bf16_t* qp = a.q + ((lane_row0 + tok[x]) * c.n_q_heads + (int64_t)g * G + head[x]) * kHeadDim + h * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 v = *reinterpret_cast<const u32x4*>(qp + j * 16);
      if (!real[x]) v = (u32x4){0u, 0u, 0u, 0u};
      qf[x][j] = as_bf16x8(v);
    }
  }
  const int wave_row0 = wave * NB * 32, wave_row1 = min(rows, wave_row0 + NB * 32) - 1;
  const bool working = wave_row0 < rows;
  const int sees_first = working ? pos0 + wave_row0 / G : -1;  // the last key that all of the wavefront's rows see
  const int sees_last = working ? pos0 + wave_row1 / G : -1;   // and that any of them sees

  // Keys and values of a step to LDS: every wavefront brings 16 tokens of each, 16 bytes a lane.
  //   keys: [64][16 chunks], chunk x of row r at x ^ r % 16, so that 32 rows at one chunk spread over the banks
  //   values by channel: the four page tiles as they stand; by token: [64][16 chunks], chunk x of row r at x ^ 2 (r % 8)
  const int64_t head_off = (int64_t)g * c.stride_head;
  int page[4], slot[4], raw[4];  // TOK: page and slot of this lane's rows of the next step; else [0] only
  const auto look_up = [&](int it) {
    if (TOK) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = it * kStep + wave * 16 + 4 * j + lane / 16;
        raw[j] = it < it1 && t < s.len ? phys_page_request(c, pl.b, page[j]) : -1;
      }
    } else {
      const int p = it * (kStep / 16) + wave;
      raw[0] = it < it1 && p * 16 < s.len ? phys_page_request(c, pl.b, p) : -1;
    }
  };
  if (TOK) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = it0 * kStep + wave * 16 + 4 * j + lane / 16;
      page[j] = t / ps;
      slot[j] = t - page[j] * ps;
    }
  }
  const int skip_pages = kStep / ps, skip_slots = kStep - skip_pages * ps;
  const auto issue = [&](int it) {  // step `it`, looked up before; looks up the next one
    unsigned char* kb = s_tiles + (it & 1) * 2 * kKeyBytes + wave * 16 * 256;
    unsigned char* vb = kb + kKeyBytes;
    if (TOK) {
      uint32_t valid = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t pp = phys_page_resolve(c, raw[j]);
        const unsigned long long ok = __ballot(pp >= 0);
#pragma unroll
        for (int x = 0; x < 4; ++x) valid |= (uint32_t)((ok >> (16 * x)) & 1u) << (4 * j + x);
        const int64_t off = pp >= 0 ? pp * c.stride_page + head_off + slot[j] * kHeadDim : 0;
        const int r = 4 * j + lane / 16;
        to_lds(c.k_pool + off + ((lane % 16) ^ r) * 8, kb + j * 1024);
        to_lds(c.v_pool + off + ((lane % 16) ^ 2 * (r % 8)) * 8, vb + j * 1024);
        slot[j] += skip_slots;
        page[j] += skip_pages;
        if (slot[j] >= ps) { slot[j] -= ps; ++page[j]; }
      }
      if (lane == 0) s_valid[it & 1][wave] = (uint16_t)valid;
    } else {
      const int64_t pp = phys_page_resolve(c, raw[0]);
      const int left = s.len - (it * kStep + wave * 16);
      if (lane == 0) s_valid[it & 1][wave] = pp < 0 || left <= 0 ? 0 : left >= 16 ? 0xffffu : (uint16_t)((1u << left) - 1);
      const int64_t off = pp >= 0 ? pp * c.stride_page + head_off : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        to_lds(c.k_pool + off + (4 * j + lane / 16) * kHeadDim + ((lane % 16) ^ (4 * j + lane / 16)) * 8, kb + j * 1024);
        to_lds(c.v_pool + off + j * 512 + lane * 8, vb + j * 1024);
      }
    }
    look_up(it + 1);
  };

  f32x16 O[NB][4];
  float m[NB], l[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    m[x] = kNegBig;
    l[x] = 0.f;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[x][cb][i] = 0.f;
  }
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  // token of the tile whose keys this lane reads as row `col` of a product: bits 2 and 3 swapped
  const int key_row = (col & 0x13) | (col & 4) << 1 | (col & 8) >> 1;

  const auto products = [&](const unsigned char* kb, int u, f32x16 (&S)[NB]) {
    const unsigned char* row = kb + (u * 32 + key_row) * 256;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bf16x8 kf = as_bf16x8(*reinterpret_cast<const u32x4*>(row + (((2 * j + h) ^ (key_row & 15)) * 16)));
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        const f32x16 zero = {};
        S[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[x][j], j == 0 ? zero : S[x], 0, 0, 0);
      }
    }
  };
  // channels 32 cb + col, tokens 32 u + 16 x + 8 h + 0..7
  const auto value_part = [&](const unsigned char* vb, int u, int x, int cb) {
    if (TOK) {
      const int i = lane % 16, chunk = (32 * cb + 16 * (lane / 16 % 2)) / 8 + i % 4 / 2;
      u32x2 w[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = 32 * u + 16 * x + 8 * h + 4 * y + i / 4;
        w[y] = lds_columns(vb + r * 256 + ((chunk ^ 2 * (r % 8)) * 16) + i % 2 * 8);
      }
      return (u32x4){w[0].x, w[0].y, w[1].x, w[1].y};
    }
    return *reinterpret_cast<const u32x4*>(vb + (2 * u + x) * 4096 + (32 * cb + col) * 32 + h * 16);
  };

  const auto unit = [&](const unsigned char* kb, const unsigned char* vb, int u, int key0, bool masked, uint32_t ok) {
    f32x16 S[NB];
    products(kb, u, S);
    if (masked) {
#pragma unroll
      for (int x = 0; x < NB; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int t = 16 * (i / 8) + 8 * h + i % 8;
          if (!((ok >> t) & 1u) || key0 + t > last[x]) S[x][i] = -INFINITY;
        }
    }
    u32x4 pf[NB][2];
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      float mx = S[x][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, S[x][i]);
      const SwapPair sw = swap_rows32(__float_as_uint(mx));
      mx = fmaxf(__uint_as_float(sw.a), __uint_as_float(sw.b)) * sc;
      if (__any(mx > m[x] + kLazy)) {
        const float mn = mx > m[x] + kLazy ? mx : m[x];
        const float alpha = fast_exp2(m[x] - mn);
        m[x] = mn;
        l[x] *= alpha;
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) O[x][cb] *= alpha;
      }
      float p[16], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = fast_exp2(fmaf(S[x][i], sc, -m[x]));
        sum += p[i];
      }
      l[x] += sum;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        pf[x][y] = (u32x4){pack_bf16x2(p[8 * y], p[8 * y + 1]), pack_bf16x2(p[8 * y + 2], p[8 * y + 3]),
                           pack_bf16x2(p[8 * y + 4], p[8 * y + 5]), pack_bf16x2(p[8 * y + 6], p[8 * y + 7])};
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        const u32x4 vf = value_part(vb, u, y, cb);
#pragma unroll
        for (int x = 0; x < NB; ++x)
          O[x][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf), as_bf16x8(pf[x][y]), O[x][cb], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
  };
  // What lies where no token is may be anything, and 0 x NaN is not 0: such values are cleared in LDS.
  const auto clear_values = [&](unsigned char* vb, unsigned long long valid) {
    for (int i = threadIdx.x; i < kStep * (kHeadDim / 8); i += kChunkT) {
      if (TOK) {
        if (!((valid >> (i / 16)) & 1ull)) *reinterpret_cast<u32x4*>(vb + i * 16) = (u32x4){0u, 0u, 0u, 0u};
      } else {  // eight tokens of a channel
        const uint32_t bits = (uint32_t)(valid >> (i / 256 * 16 + i % 2 * 8)) & 0xffu;
        if (bits == 0xffu) continue;
        u32x4* at = reinterpret_cast<u32x4*>(vb + i * 16);
        u32x4 v = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] &= (((bits >> (2 * e)) & 1u) ? 0x0000ffffu : 0u) | (((bits >> (2 * e + 1)) & 1u) ? 0xffff0000u : 0u);
        *at = v;
      }
    }
  };

  look_up(it0);
  if (it0 < it1) issue(it0);
  for (int it = it0; it < it1; ++it) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // this wavefront's share of the step has landed
    __syncthreads();                                             // everyone's has, and the other buffer is free
    unsigned char* kb = s_tiles + (it & 1) * 2 * kKeyBytes;
    unsigned char* vb = kb + kKeyBytes;
    const u32x2 bits = *reinterpret_cast<const u32x2*>(s_valid[it & 1]);
    const unsigned long long valid = (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)bits.y) << 32 |
                                     (uint32_t)__builtin_amdgcn_readfirstlane((int)bits.x);
    if (valid != ~0ull) {
      clear_values(vb, valid);
      __syncthreads();
    }
    if (it + 1 < it1) issue(it + 1);
    if (!working || it * kStep > sees_last) continue;
    const bool masked = valid != ~0ull || it * kStep + kStep - 1 > sees_first;
#pragma unroll 1
    for (int u = 0; u < 2; ++u) unit(kb, vb, u, it * kStep + 32 * u, masked, (uint32_t)(valid >> (32 * u)));
  }

#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const SwapPair sw = swap_rows32(__float_as_uint(l[x]));
    const float sum = __uint_as_float(sw.a) + __uint_as_float(sw.b);
    if (!real[x]) continue;
    if (pl.parts > 1) {
      float* o = a.partial + (((int64_t)at * c.n_kv_heads + g) * kRows + (wave * NB + x) * 32 + col) * kRowStride;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 16; i += 2)
          *reinterpret_cast<float2*>(o + 32 * cb + 8 * (i / 4) + 4 * h + i % 4) = make_float2(O[x][cb][i], O[x][cb][i + 1]);
      if (h == 0) *reinterpret_cast<float2*>(o + kHeadDim) = make_float2(m[x], sum);
    } else {
      const int64_t row = (lane_row0 + tok[x]) * c.n_q_heads + (int64_t)g * G + head[x];
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      bf16_t* o = a.out + row * kHeadDim;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<u32x2*>(o + 32 * cb + 2 * i + 4 * h) =
              (u32x2){pack_bf16x2(O[x][cb][i] * inv, O[x][cb][i + 1] * inv), pack_bf16x2(O[x][cb][i + 2] * inv, O[x][cb][i + 3] * inv)};
      if (a.out_lse && h == 0) a.out_lse[row] = sum > 0.f ? (m[x] + __log2f(sum)) * kLn2 : -INFINITY;
    }
  }
}

// The parts of a tile joined: a wavefront per row, a lane per two channels.
__global__ __launch_bounds__(256) void chunk_merge_kernel(CacheView c, ChunkAttendArgs a, int tile_rows) {
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads;
  const int size = chunk_size_for(c, a);
  if (size == kChunkWhole) return;
  ChunkPlace pl;
  if (!chunk_place(c, a, size, at, pl) || pl.parts == 1) return;
  const ChunkSeq s = chunk_seq(c, a.ch, pl.b);
  const int G = c.group, t0 = pl.tile * a.tile_tokens, rows = min(a.tile_tokens, s.n - t0) * G;
  const int lane = threadIdx.x % kWave;
  // the tile's parts share its rows
  for (int r = pl.part + pl.parts * (threadIdx.x / kWave + 4 * blockIdx.y); r < rows; r += pl.parts * 4 * gridDim.y) {
    const float* p = a.partial + (((int64_t)pl.first * c.n_kv_heads + g) * tile_rows + r) * kRowStride;
    const int64_t next = (int64_t)c.n_kv_heads * tile_rows * kRowStride;
    float m = kNegBig;
    for (int i = 0; i < pl.parts; ++i) m = fmaxf(m, p[i * next + kHeadDim]);
    float l = 0.f, x = 0.f, y = 0.f;
    for (int i = 0; i < pl.parts; ++i) {
      const float2 ml = *reinterpret_cast<const float2*>(p + i * next + kHeadDim);
      const float2 o = *reinterpret_cast<const float2*>(p + i * next + 2 * lane);
      const float w = fast_exp2(ml.x - m);
      l = fmaf(ml.y, w, l);
      x = fmaf(o.x, w, x);
      y = fmaf(o.y, w, y);
    }
    const int t = r / G;
    const int64_t row = (int64_t)(s.row + t0 + t) * c.n_q_heads + (int64_t)g * G + r - t * G;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<uint32_t*>(a.out + row * kHeadDim + 2 * lane) = pack_bf16x2(x * inv, y * inv);
    if (a.out_lse && lane == 0) a.out_lse[row] = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
  }
}

ChunkPlan plan_chunk_attend(const CacheView& c, int n_tokens) {
  ChunkPlan p;
  // 64 rows to a wavefront read LDS half as often for the same products; 32 where a sequence has few rows on average
  const int64_t rows = (int64_t)n_tokens * c.group;
  p.blocks = rows > 128ll * c.batch ? 2 : 1;
  p.tile_rows = 128 * p.blocks;
  p.tile_tokens = p.tile_rows / c.group;
  p.target = 512;
  const int64_t at_least = ((int64_t)n_tokens + p.tile_tokens - 1) / p.tile_tokens * c.n_kv_heads;
  int64_t tiles = ((int64_t)n_tokens / p.tile_tokens + c.batch);
  if (tiles > n_tokens) tiles = n_tokens;
  tiles *= c.n_kv_heads;
  p.cuts = at_least < p.target;
  p.workgroups = p.cuts && tiles < p.target ? p.target : tiles;
  p.total_bytes = p.cuts ? (size_t)ROCKETKV_WS_HEADER_BYTES + (size_t)p.target * p.tile_rows * kRowStride * sizeof(float) : 0;
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
  a.partial = plan.cuts ? reinterpret_cast<float*>(static_cast<char*>(ws) + ROCKETKV_WS_HEADER_BYTES) : nullptr;
  a.tile_tokens = plan.tile_tokens;
  a.target = plan.target;
  const dim3 grid((unsigned)plan.workgroups), block(kChunkT);
  const size_t lds = 2 * 2 * kKeyBytes;
  if (plan.blocks == 1) {
    if (c.v_token_major) hipLaunchKernelGGL((chunk_attend_kernel<true, 1>), grid, block, lds, st, c, a);
    else hipLaunchKernelGGL((chunk_attend_kernel<false, 1>), grid, block, lds, st, c, a);
  } else {
    if (c.v_token_major) hipLaunchKernelGGL((chunk_attend_kernel<true, 2>), grid, block, lds, st, c, a);
    else hipLaunchKernelGGL((chunk_attend_kernel<false, 2>), grid, block, lds, st, c, a);
  }
  if (plan.cuts) {
    const unsigned wgs = (unsigned)(plan.workgroups < plan.target ? plan.workgroups : plan.target);
    hipLaunchKernelGGL(chunk_merge_kernel, dim3(wgs), dim3(256), 0, st, c, a, plan.tile_rows);
  }
  return hipGetLastError();
}

}  // namespace rkv
