// Rotary positions, alone and on the way of new tokens into the cache.
//
// A position p turns channel pair i of a head by the angle p * inv_freq[i]:
//   (x, y) -> s * (x cos - y sin, y cos + x sin)
// where the pairs are (2i, 2i+1) or (i, i + rot_dim/2) of the leading rot_dim channels; the others pass through.
// Angles of far positions need more than 24 bits (position 131071 at the highest frequency is 20861 turns), so they are
// formed as turns in 64 bits, reduced there, and only what is left of a turn goes to 32.
//
// Both kernels are bound by memory: every head row is read and written once.  What would cost more than that, the sines,
// is computed once per token and pair into LDS and used by all heads a workgroup handles.
#include "common.h"
#include "quantise.h"

namespace rkv {

namespace {

constexpr int kRopeT = 256;                 // threads
constexpr int kRowLanes = kHeadDim / 8;     // lanes that hold a head row, eight channels each
constexpr int kRowsPerPass = kRopeT / kRowLanes;
constexpr int kBlockTokens = 32;            // tokens whose sines are in LDS at a time
constexpr int kRowsInFlight = 4;            // rows a thread has requested at once
constexpr int kQueryRows = 128;             // of a block of queries of few tokens
constexpr int kFewBlocks = 432;             // workgroups with tokens below which blocks of pages become smaller

typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));

struct Eight {
  float x[8];
};
__device__ __forceinline__ Eight unpack8(uint4 v) {
  Eight r;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.x[2 * i] = bf16lo_to_f32(w[i]);
    r.x[2 * i + 1] = bf16hi_to_f32(w[i]);
  }
  return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 pair_bf16 __attribute__((ext_vector_type(2)));
  typedef float pair_f32 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((pair_f32){lo, hi}, pair_bf16));
}

// STREAM: past the caches.  138 -> 132 us for 32768 tokens of 40 heads; queries on the way into the cache, which is what
// reads them next, lose by it (712 -> 720 us for 131072 tokens).
template <bool STREAM>
__device__ __forceinline__ void st16(bf16_t* p, uint4 v) {
  const rope_u32x4 x = {v.x, v.y, v.z, v.w};
  if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<rope_u32x4*>(p));
  else *reinterpret_cast<rope_u32x4*>(p) = x;
}

// s * (cos, sin) of the angles of tokens [0, n) at `pos_of(token)`, all threads of the workgroup
template <class Pos>
__device__ __forceinline__ void fill_turns(const RopeView& r, int n, const Pos& pos_of, float2* s_cs) {
  const int half = r.rot_dim / 2;
  for (int i = threadIdx.x; i < n * half; i += kRopeT) {
    const int t = i / half, p = i - t * half;
    const double turns = (double)pos_of(t) * (r.inv_freq[p] * 0.15915494309189535);  // angle / 2 pi
    float sn, cs;
    sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
    s_cs[t * half + p] = make_float2(cs * r.scale, sn * r.scale);
  }
}

// What a lane needs of a row before it can turn its eight channels: the channels, and in the half layout the ones half a
// rotation away (a second load of the same lines).  Requested first, turned later, so that rows overlap.
struct RowPart {
  uint4 own, far;
};
// ODD: half a rotation is no multiple of eight channels, and the partners are not eight neighbours at one.
template <bool ODD>
__device__ __forceinline__ RowPart request_row(const RopeView& r, const bf16_t* row, int c0) {
  RowPart p;
  p.own = ld16<false>(row + c0);
  p.far = make_uint4(0, 0, 0, 0);
  const int half = r.rot_dim / 2;
  if (!r.interleaved && c0 < r.rot_dim) {
    if (!ODD) {
      p.far = ld16<false>(row + (c0 < half ? c0 + half : c0 - half));
    } else {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = c0 + e;
        w[e] = c < r.rot_dim ? row[c < half ? c + half : c - half] : 0;
      }
      p.far = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
  }
  return p;
}
inline bool rope_is_odd(const RopeView& r) { return !r.interleaved && r.rot_dim % 16 != 0; }
__device__ __forceinline__ Eight turn8(const RopeView& r, const RowPart& p, const float2* cs, int c0) {
  const Eight a = unpack8(p.own);
  Eight out;
  float (&y)[8] = out.x;
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = c0 + 2 * i < r.rot_dim;
      const float2 t = cs[in ? c0 / 2 + i : 0];
      y[2 * i] = in ? a.x[2 * i] * t.x - a.x[2 * i + 1] * t.y : a.x[2 * i];
      y[2 * i + 1] = in ? a.x[2 * i + 1] * t.x + a.x[2 * i] * t.y : a.x[2 * i + 1];
    }
  } else {
    const Eight f = unpack8(p.far);
    const int half = r.rot_dim / 2;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = c0 + e;
      const bool low = c < half, in = c < r.rot_dim;
      const float2 t = cs[low ? c : in ? c - half : 0];
      y[e] = in ? a.x[e] * t.x + (low ? -f.x[e] : f.x[e]) * t.y : a.x[e];
    }
  }
  return out;
}
// rounded to bf16 once, at the end
__device__ __forceinline__ uint4 turn_row(const RopeView& r, const RowPart& p, const float2* cs, int c0) {
  const Eight y = turn8(r, p, cs, c0);
  return make_uint4(pack2(y.x[0], y.x[1]), pack2(y.x[2], y.x[3]), pack2(y.x[4], y.x[5]), pack2(y.x[6], y.x[7]));
}

// `n` tokens of `heads` heads each, from x (rows of x_stride elements a token) to y, by the whole workgroup; the
// tokens' turns are in s_cs.  Every lane has read all it needs of a row before the wavefront stores into it, and a row
// belongs to one wavefront, so x and y may be the same memory.
template <bool STREAM, bool ODD>
__device__ __forceinline__ void turn_heads(const RopeView& r, const bf16_t* x, int64_t x_stride, bf16_t* y, int64_t y_stride,
                                           int n, int heads, const float2* s_cs) {
  const int c0 = threadIdx.x % kRowLanes * 8, half = r.rot_dim / 2;
  const int rows = n * heads;
  for (int i0 = threadIdx.x / kRowLanes; i0 < rows; i0 += kRowsPerPass * kRowsInFlight) {
    RowPart p[kRowsInFlight];
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      const int i = i0 + u * kRowsPerPass, t = i / heads, h = i - t * heads;
      if (i < rows) p[u] = request_row<ODD>(r, x + t * x_stride + h * kHeadDim, c0);
    }
#pragma unroll
    for (int u = 0; u < kRowsInFlight; ++u) {
      const int i = i0 + u * kRowsPerPass, t = i / heads, h = i - t * heads;
      if (i < rows) {
        const uint4 o = turn_row(r, p[u], s_cs + t * half, c0);
        st16<STREAM>(y + t * y_stride + h * kHeadDim + c0, o);
      }
    }
  }
}

template <bool ODD>
__global__ __launch_bounds__(kRopeT) void rope_kernel(RopeView r, const int32_t* __restrict__ positions, int n_tokens,
                                                     int heads, const bf16_t* x, int64_t x_stride, bf16_t* y,
                                                     int64_t y_stride, int per_wg) {
  extern __shared__ float2 s_cs[];
  const int t0 = blockIdx.x * per_wg, n = min(per_wg, n_tokens - t0);
  fill_turns(r, n, [&](int t) { return positions[t0 + t]; }, s_cs);
  __syncthreads();
  turn_heads<true, ODD>(r, x + t0 * x_stride, x_stride, y + t0 * y_stride, y_stride, n, heads, s_cs);
}

// What a chunk brings to sequence b.
struct NewTokens {
  int row, n;    // its rows in the packed tensors
  int old;       // tokens the sequence held
  bool room;     // they fit
};
__device__ __forceinline__ NewTokens new_tokens(const CacheView& c, const ChunkView& ch, int b) {
  NewTokens s;
  s.row = chunk_first(ch, b);
  s.n = chunk_rows(ch, b);
  s.old = (int)use_late((uint32_t)c.seq_lens[b]);  // here, not later: the length is stored anew once all have it
  s.room = s.old >= 0 && (int64_t)s.old + s.n <= (int64_t)c.pages_cap * c.page_size;
  return s;
}

}  // namespace

// New tokens into the cache, in one launch: the first workgroups take blocks of `pages` pages (aligned to `pages`; where that is
// eight or more, a multiple of eight, a channel's summaries leave as whole 16-byte pieces) of some heads, the others blocks of
// query rows (with the two kinds mixed instead, 131072 tokens take 797 us, so 706).  A block is worked through kBlockTokens tokens at a time: sines of the tokens, then head by head the key rows
// (turned) and the value rows to the pools and to LDS, from where a thread takes a pair of channels down the tokens of a
// page: extremes of the keys, in the order of the tokens as single appends would fold them, and the 16 values of a
// channel-major tile's row.  Quantised caches take codes instead, by token, and LDS the values these stand for.
struct AppendChunkArgs {
  ChunkView ch;
  RopeView rope;              // rot_dim 0: nothing is turned
  const int32_t* positions;   // null: a token's place in the cache
  const bf16_t *q, *k, *v;    // q null: no queries
  int64_t q_stride, k_stride, v_stride;
  bf16_t *q_out, *kmax, *kmin;  // kmax null: no summaries
  int pages, kv_wgs, heads_per_wg, head_groups, q_block;
  uint32_t* arrived;  // per sequence at read_slot(): workgroups that have read its length
  uint8_t *k_scales, *v_scales;  // of a quantised cache
};

// FMT: of a quantised cache, whose pools and strides `c` then holds; or kBf16.
template <bool ODD, int FMT>
__global__ __launch_bounds__(kRopeT) __attribute__((amdgpu_waves_per_eu(ODD || FMT != kBf16 ? 3 : 4)))
void append_chunk_kernel(CacheView c, AppendChunkArgs a) {
  extern __shared__ __align__(16) unsigned char s_mem[];
  float2* s_cs = reinterpret_cast<float2*>(s_mem);                                                    // [tokens][pairs]
  uint32_t* s_k = reinterpret_cast<uint32_t*>(s_mem + (size_t)kBlockTokens * kHeadDim / 2 * sizeof(float2));  // [tokens][64]
  uint32_t* s_v = s_k + kBlockTokens * kHeadDim / 2;
  bf16_t* s_sum = reinterpret_cast<bf16_t*>(FMT != kBf16 ? s_v : s_v + kBlockTokens * kHeadDim / 2);    // [heads][2][128][pages]
  const int tid = threadIdx.x, ps = c.page_size;
  const bool turns = a.rope.rot_dim > 0;
  const int span = a.pages * ps;  // token slots of a block of pages
  // Divided by the new tokens alone, wherever they begin inside a block: lengths of other sequences may be stored
  // anew at any time.
  const auto kv_tiles = [&](int n) { return n > 0 ? (n + span - 2) / span + 1 : 0; };
  const auto q_tiles = [&](int n) { return a.q ? (n + a.q_block - 1) / a.q_block : 0; };
  const int n_kv = a.kv_wgs * a.head_groups;
  const bool is_kv = (int)blockIdx.x < n_kv;
  int b, tile;
  if (is_kv) {
    if (!locate_tile(c.batch, blockIdx.x / a.head_groups, [&](int i) { return kv_tiles(chunk_rows(a.ch, i)); }, b, tile)) return;
  } else {
    if (!locate_tile(c.batch, blockIdx.x - n_kv, [&](int i) { return q_tiles(chunk_rows(a.ch, i)); }, b, tile)) return;
  }
  const NewTokens s = new_tokens(c, a.ch, b);

  if (!is_kv) {
    const int t0 = tile * a.q_block, n = min(a.q_block, s.n - t0), r0 = s.row + t0;
    const bf16_t* x = a.q + (int64_t)r0 * a.q_stride;
    bf16_t* y = a.q_out + (int64_t)r0 * c.n_q_heads * kHeadDim;
    if (turns) {
      fill_turns(a.rope, n, [&](int t) { return a.positions ? a.positions[r0 + t] : s.old + t0 + t; }, s_cs);
      __syncthreads();
    }
    turn_heads<false, ODD>(a.rope, x, a.q_stride, y, (int64_t)c.n_q_heads * kHeadDim, n, c.n_q_heads, s_cs);
  } else if (s.room) {
    const int g0 = (int)(blockIdx.x % a.head_groups) * a.heads_per_wg, ng = min(a.heads_per_wg, c.n_kv_heads - g0);
    const int p0 = (s.old / span + tile) * a.pages;
    const int lo = max(s.old, p0 * ps), hi = min(s.old + s.n, p0 * ps + span);  // the block's new tokens
    const int half = a.rope.rot_dim / 2, c0 = tid % kRowLanes * 8, i0 = tid / kRowLanes;
    constexpr int kPasses = kBlockTokens / kRowsPerPass;
    const int first_tb = lo < hi ? p0 * ps + (lo - p0 * ps) / kBlockTokens * kBlockTokens : hi;
    for (int tb = first_tb; tb < hi; tb += kBlockTokens) {
      const int tl = max(lo, tb), th = min(hi, tb + kBlockTokens);
      if (turns) {
        __syncthreads();  // the last block's turns have been used
        fill_turns(a.rope, th - tl, [&](int t) { const int r = s.row + tl + t - s.old; return a.positions ? a.positions[r] : tl + t; }, s_cs);
      }
      for (int gi = 0; gi < ng; ++gi) {
        const int g = g0 + gi;
        __syncthreads();  // the turns are there; the last head's rows have been used
        RowPart kp[kPasses];
        uint4 vp[kPasses];
#pragma unroll
        for (int u = 0; u < kPasses; ++u) {
          const int t = tl + i0 + u * kRowsPerPass;
          if (t < th) {
            const int64_t r = s.row + t - s.old;
            kp[u] = request_row<ODD>(a.rope, a.k + r * a.k_stride + g * kHeadDim, c0);
            vp[u] = ld16<true>(a.v + r * a.v_stride + g * kHeadDim + c0);
          }
        }
#pragma unroll
        for (int u = 0; u < kPasses; ++u) {
          const int i = i0 + u * kRowsPerPass, t = tl + i;
          if constexpr (FMT != kBf16) {
            if (t < th) {
              const Codes8 k = turns ? quantise8<FMT>(turn8(a.rope, kp[u], s_cs + i * half, c0).x) : quantise8<FMT>(kp[u].own);
              const Codes8 v = quantise8<FMT>(vp[u]);
              if (a.kmax) *reinterpret_cast<uint4*>(s_k + i * (kHeadDim / 2) + c0 / 2) = restore8<FMT>(k.codes, k.scale);
              const int64_t pp = phys_page(c, b, t / ps);
              if (pp >= 0) {
                const int64_t at = pp * c.stride_page + g * c.stride_head + t % ps;
                store_codes<FMT>(c.k_pool, a.k_scales, at, c0 / 8, k);
                store_codes<FMT>(c.v_pool, a.v_scales, at, c0 / 8, v);
              }
            }
          } else if (t < th) {
            const uint4 k = turns ? turn_row(a.rope, kp[u], s_cs + i * half, c0) : kp[u].own;
            *reinterpret_cast<uint4*>(s_k + i * (kHeadDim / 2) + c0 / 2) = k;
            if (!c.v_token_major) *reinterpret_cast<uint4*>(s_v + i * (kHeadDim / 2) + c0 / 2) = vp[u];
            const int64_t pp = phys_page(c, b, t / ps);
            if (pp >= 0) {
              const int64_t at = pp * c.stride_page + g * c.stride_head + (int64_t)(t % ps) * kHeadDim + c0;
              *reinterpret_cast<uint4*>(c.k_pool + at) = k;
              if (c.v_token_major) *reinterpret_cast<uint4*>(c.v_pool + at) = vp[u];
            }
          }
        }
        __syncthreads();
        // a pair of channels down the tokens of a page
        const int first = tl / ps, last = (th - 1) / ps;
        const int n_sum = a.kmax ? (last - first + 1) * (kHeadDim / 2) : 0;
        const int n_val = c.v_token_major ? 0 : (last - first + 1) * (kHeadDim / 2);
        for (int i = tid; i < n_sum + n_val; i += kRopeT) {
          const bool sums = i < n_sum;
          const int j = sums ? i : i - n_sum;
          const int p = first + j / (kHeadDim / 2), cp = j % (kHeadDim / 2);
          const int t0 = max(tl, p * ps), t1 = min(th, (p + 1) * ps);
          if (sums) {
            bf16_t* smax = s_sum + ((gi * 2 * kHeadDim + 2 * cp) * a.pages + p - p0);
            bf16_t* smin = smax + kHeadDim * a.pages;
            const int64_t o = (((int64_t)b * c.n_kv_heads + g) * kHeadDim + 2 * cp) * c.pages_cap + p;
            bf16_t mx[2], mn[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const bf16_t x = (bf16_t)(s_k[(t0 - tl) * (kHeadDim / 2) + cp] >> (16 * e));
              mx[e] = mn[e] = x;
              if (t0 % ps != 0) {  // the page was begun before: by older tokens, or by this launch's last block of tokens
                const bf16_t ox = t0 == s.old ? a.kmax[o + e * c.pages_cap] : smax[e * a.pages];
                const bf16_t on = t0 == s.old ? a.kmin[o + e * c.pages_cap] : smin[e * a.pages];
                if (!(bf16_to_f32(x) > bf16_to_f32(ox))) mx[e] = ox;
                if (!(bf16_to_f32(x) < bf16_to_f32(on))) mn[e] = on;
              }
            }
            for (int t = t0 + 1; t < t1; ++t) {
              const uint32_t w = s_k[(t - tl) * (kHeadDim / 2) + cp];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const bf16_t x = (bf16_t)(w >> (16 * e));
                if (bf16_to_f32(x) > bf16_to_f32(mx[e])) mx[e] = x;
                if (bf16_to_f32(x) < bf16_to_f32(mn[e])) mn[e] = x;
              }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              smax[e * a.pages] = mx[e];
              smin[e * a.pages] = mn[e];
            }
          } else {
            const int64_t pp = phys_page(c, b, p);
            if (pp < 0) continue;
            bf16_t* dst = c.v_pool + pp * c.stride_page + g * c.stride_head + (int64_t)2 * cp * kAttnPage;
            const uint32_t* col = s_v + (t0 - tl) * (kHeadDim / 2) + cp;
            if (t1 - t0 == kAttnPage) {
              uint32_t lo16[kAttnPage / 2], hi16[kAttnPage / 2];
#pragma unroll
              for (int x = 0; x < kAttnPage / 2; ++x) {
                const uint32_t w0 = col[2 * x * (kHeadDim / 2)], w1 = col[(2 * x + 1) * (kHeadDim / 2)];
                lo16[x] = (w0 & 0xffffu) | w1 << 16;
                hi16[x] = w0 >> 16 | (w1 & 0xffff0000u);
              }
              uint4* d = reinterpret_cast<uint4*>(dst);
              d[0] = make_uint4(lo16[0], lo16[1], lo16[2], lo16[3]);
              d[1] = make_uint4(lo16[4], lo16[5], lo16[6], lo16[7]);
              d[2] = make_uint4(hi16[0], hi16[1], hi16[2], hi16[3]);
              d[3] = make_uint4(hi16[4], hi16[5], hi16[6], hi16[7]);
            } else {  // the page's other slots stay as they are
              for (int t = t0; t < t1; ++t) {
                const uint32_t w = col[(t - t0) * (kHeadDim / 2)];
                dst[t % ps] = (bf16_t)w;
                dst[kAttnPage + t % ps] = (bf16_t)(w >> 16);
              }
            }
          }
        }
      }
    }
    if (a.kmax && lo < hi) {
      __syncthreads();
      const int first = lo / ps - p0, last = (hi - 1) / ps - p0;  // pages that took in a token
      const int groups = (a.pages + 7) / 8;
      for (int i = tid; i < ng * 2 * kHeadDim * groups; i += kRopeT) {
        const int pg = i % groups * 8, row = i / groups;  // row: (head, extreme, channel)
        const int chn = row % kHeadDim, gi = row / (2 * kHeadDim);
        bf16_t* out = (row / kHeadDim % 2 ? a.kmin : a.kmax) + (((int64_t)b * c.n_kv_heads + g0 + gi) * kHeadDim + chn) * c.pages_cap + p0 + pg;
        const bf16_t* in = s_sum + (int64_t)row * a.pages + pg;
        if (first <= pg && pg + 7 <= last) {
          *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(in);
        } else {
          for (int e = max(0, first - pg); e < 8 && pg + e <= last; ++e) out[e] = in[e];
        }
      }
    }
  }
  // The last of a sequence's workgroups to have read its length stores the new one.
  __syncthreads();
  if (tid == 0 && s.room) {
    const uint32_t all = (uint32_t)(kv_tiles(s.n) * a.head_groups + q_tiles(s.n));
    uint32_t* n = a.arrived + read_slot(c, b);
    if (__hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1) {
      clear_reads(a.arrived, read_slot(c, b));
      c.seq_lens[b] = s.old + s.n;
    }
  }
}

// Keys and values that come turned into a quantised cache: sixteen lanes take a page, token by token, eight channels each, so
// the extremes of its keys stay in registers, and only they pass through LDS, a workgroup's pages next to each other.
// 32768 tokens of 8 heads into 4 bits, 170 MB read and written: 44 us, 3.9 TB/s; 81 by the kernel above, which takes the rows
// through LDS for the extremes.
constexpr int kPutPages = kRopeT / kRowLanes;
constexpr int kPutRows = 4;  // tokens a lane has requested at once

template <int FMT>
__global__ __launch_bounds__(kRopeT) void put_chunk_kernel(CacheView c, AppendChunkArgs a) {
  __shared__ __align__(16) bf16_t s_sum[2 * kHeadDim * kPutPages];  // [extreme][channel][page]
  const int tid = threadIdx.x, ps = c.page_size, span = kPutPages * ps, g = blockIdx.x % c.n_kv_heads;
  const auto tiles = [&](int n) { return n > 0 ? (n + span - 2) / span + 1 : 0; };
  int b, tile;
  if (!locate_tile(c.batch, blockIdx.x / c.n_kv_heads, [&](int i) { return tiles(chunk_rows(a.ch, i)); }, b, tile)) return;
  const NewTokens s = new_tokens(c, a.ch, b);
  if (s.room) {
    const int p0 = (s.old / span + tile) * kPutPages, p = p0 + tid / kRowLanes, lane16 = tid % kRowLanes;
    const int lo = max(s.old, p * ps), hi = min(s.old + s.n, (p + 1) * ps);
    const int64_t pp = lo < hi ? phys_page(c, b, p) : -1, tok = pp * c.stride_page + g * c.stride_head - p * ps;
    const int64_t sums = (((int64_t)b * c.n_kv_heads + g) * kHeadDim + lane16 * 8) * c.pages_cap + p;
    float mx[8], mn[8];
    bool begun = lo % ps != 0 && lo < hi;  // by older tokens
    if (a.kmax && begun)
#pragma unroll
      for (int e = 0; e < 8; ++e) mx[e] = bf16_to_f32(a.kmax[sums + e * c.pages_cap]), mn[e] = bf16_to_f32(a.kmin[sums + e * c.pages_cap]);
    for (int t0 = lo; t0 < hi; t0 += kPutRows) {
      uint4 k[kPutRows], v[kPutRows];
#pragma unroll
      for (int u = 0; u < kPutRows; ++u) {
        const int64_t r = s.row + min(t0 + u, hi - 1) - s.old;
        k[u] = ld16<true>(a.k + r * a.k_stride + g * kHeadDim + lane16 * 8);
        v[u] = ld16<true>(a.v + r * a.v_stride + g * kHeadDim + lane16 * 8);
      }
#pragma unroll
      for (int u = 0; u < kPutRows; ++u) {
        if (t0 + u >= hi) break;
        const Codes8 kc = quantise8<FMT>(k[u]), vc = quantise8<FMT>(v[u]);
        if (pp >= 0) {
          store_codes<FMT>(c.k_pool, a.k_scales, tok + t0 + u, lane16, kc);
          store_codes<FMT>(c.v_pool, a.v_scales, tok + t0 + u, lane16, vc);
        }
        if (a.kmax) {
          const Eight x = unpack8(restore8<FMT>(kc.codes, kc.scale));
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (!begun || x.x[e] > mx[e]) mx[e] = x.x[e];
            if (!begun || x.x[e] < mn[e]) mn[e] = x.x[e];
          }
          begun = true;
        }
      }
    }
    if (a.kmax) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        bf16_t* to = s_sum + (lane16 * 8 + e) * kPutPages + tid / kRowLanes;
        to[0] = (bf16_t)(__float_as_uint(mx[e]) >> 16);
        to[kHeadDim * kPutPages] = (bf16_t)(__float_as_uint(mn[e]) >> 16);
      }
      __syncthreads();
      const int first = max(s.old, p0 * ps) / ps - p0, last = (min(s.old + s.n, (p0 + kPutPages) * ps) - 1) / ps - p0;  // pages that took in a token
      for (int i = tid; i < 2 * kHeadDim * (kPutPages / 8); i += kRopeT) {
        const int pg = i % (kPutPages / 8) * 8, row = i / (kPutPages / 8);
        bf16_t* out = (row / kHeadDim ? a.kmin : a.kmax) + (((int64_t)b * c.n_kv_heads + g) * kHeadDim + row % kHeadDim) * c.pages_cap + p0 + pg;
        const bf16_t* in = s_sum + row * kPutPages + pg;
        if (first <= pg && pg + 7 <= last) *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(in);
        else
          for (int e = max(0, first - pg); e < 8 && pg + e <= last; ++e) out[e] = in[e];
      }
    }
  }
  // The last of a sequence's workgroups to have read its length stores the new one.
  __syncthreads();
  if (tid == 0 && s.room) {
    uint32_t* n = a.arrived + read_slot(c, b);
    if (__hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(tiles(s.n) * c.n_kv_heads) - 1) {
      clear_reads(a.arrived, read_slot(c, b));
      c.seq_lens[b] = s.old + s.n;
    }
  }
}

hipError_t launch_rope(const RopeView& r, const int32_t* positions, int n_tokens, int n_heads, const bf16_t* x,
                       int64_t x_stride, bf16_t* y, int64_t y_stride, hipStream_t st) {
  if (n_tokens == 0 || n_heads == 0) return hipSuccess;
  int per_wg = (n_tokens + 2047) / 2048;
  if (per_wg > kBlockTokens) per_wg = kBlockTokens;
  const size_t lds = (size_t)per_wg * (r.rot_dim / 2) * sizeof(float2);
  hipLaunchKernelGGL(rope_is_odd(r) ? rope_kernel<true> : rope_kernel<false>, dim3((n_tokens + per_wg - 1) / per_wg),
                     dim3(kRopeT), lds, st, r, positions, n_tokens, n_heads, x, x_stride, y, y_stride, per_wg);
  return hipGetLastError();
}

namespace {

template <int FMT>
hipError_t launch_append_any(const CacheView& c, uint8_t* k_scales, uint8_t* v_scales, const ChunkView& ch, const RopeView& r,
                             const int32_t* positions, const bf16_t* q, int64_t q_stride, bf16_t* q_out, const bf16_t* k,
                             int64_t k_stride, const bf16_t* v, int64_t v_stride, bf16_t* kmax, bf16_t* kmin, void* ws,
                             hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  AppendChunkArgs a;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.ch = ch;
  a.rope = r;
  a.positions = positions;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.kmax = kmax;
  a.kmin = kmin;
  a.arrived = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + ROCKETKV_WS_HEADER_BYTES / 2);
  if constexpr (FMT != kBf16) {
    if (r.rot_dim == 0 && !q) {
      const int64_t blocks = (int64_t)ch.n_tokens / (kPutPages * c.page_size) + 2ll * c.batch;
      const int64_t wgs = (blocks < ch.n_tokens ? blocks : ch.n_tokens) * c.n_kv_heads;
      if (wgs * kRopeT <= 0xffffffffll) {  // (what a grid may have)
        hipLaunchKernelGGL(put_chunk_kernel<FMT>, dim3((unsigned)wgs), dim3(kRopeT), 0, st, c, a);
        return hipGetLastError();
      }
    }
  }
  // Blocks of about 128 tokens; smaller ones where there are few.
  int pages = ((128 + c.page_size - 1) / c.page_size + 7) / 8 * 8;
  if (pages > 32) pages = 32;  // 16 KiB of summaries a head
  const auto blocks = [&](int pages) {  // n tokens touch at most n / span + 2, and no more than there are tokens
    const int64_t x = (int64_t)ch.n_tokens / (pages * c.page_size) + 2ll * c.batch;
    return (int)(x < ch.n_tokens ? x : ch.n_tokens);
  };
  while (pages > 8 && (int64_t)blocks(pages) * c.n_kv_heads < 1024) pages -= 8;
  // A block's tokens come kBlockTokens at a time, one lot after the other: fewer pages, where that would leave the chip idle, a
  // block more of each sequence than its tokens fill taken for half empty.  bf16, 32 heads over 8, pages of 16, with a launch that
  // sets the lengths back, us in blocks of 8 and of 4 pages by the workgroups of 8: 48.2 and 41.6 (5000 tokens, 320), 49.2 and
  // 48.0 (6000, 376), 44.4 and 36.6 (300 of each of 16 sequences, 424), but 49.5 and 53.7 (7000, 440), 57.5 and 61.8 (8192, 520),
  // 62.9 and 67.9 (10000, 632).  In blocks of 8 pages and of those taken: 64 of each of 16 23 and 16.5, 159 of each of 2 25 and
  // 14.4, 2048 in pages of 64 129 and 28; into 8 bits 4000 of 64 heads in 2 pages 56, in 4 50.
  const auto filled = [&](int pages) {
    const int64_t x = (int64_t)ch.n_tokens / (pages * c.page_size) + c.batch;
    return x < ch.n_tokens ? x : ch.n_tokens;
  };
  while (pages > 1 && pages * c.page_size > kBlockTokens && filled(pages) * c.n_kv_heads < kFewBlocks) pages /= 2;
  a.pages = pages;
  a.kv_wgs = blocks(pages);
  a.heads_per_wg = c.n_kv_heads < 4 ? c.n_kv_heads : 4;
  while (a.heads_per_wg > 1 && (int64_t)a.kv_wgs * ((c.n_kv_heads + a.heads_per_wg - 1) / a.heads_per_wg) < 1024) a.heads_per_wg /= 2;
  while (a.heads_per_wg > 1 && a.heads_per_wg * 2 * kHeadDim * pages * 2 > 32 * 1024) a.heads_per_wg /= 2;
  a.head_groups = (c.n_kv_heads + a.heads_per_wg - 1) / a.heads_per_wg;
  // Queries in 2048 blocks at most, and fewer of up to kQueryRows rows: workgroups that find their places and form sines for a
  // token or two come in more rounds.  (2048 tokens of 32 heads into 8 bits 30 us so, 42 in 2048 blocks; 600 17, 20; 4942 of each
  // of 2 of 8 heads 58, 64; but 4000 of 64 heads in blocks of 512 rows 35, of 128 33.)
  const int few_tokens = kQueryRows / c.n_q_heads < 1 ? 1 : kQueryRows / c.n_q_heads;
  a.q_block = (ch.n_tokens + 511) / 512 < few_tokens ? (ch.n_tokens + 511) / 512 : few_tokens;
  if (a.q_block < (ch.n_tokens + 2047) / 2048) a.q_block = (ch.n_tokens + 2047) / 2048;
  if (a.q_block > kBlockTokens) a.q_block = kBlockTokens;
  const int64_t q_blocks = q ? (int64_t)ch.n_tokens / a.q_block + c.batch : 0;
  const int q_wgs = (int)(q_blocks < ch.n_tokens ? q_blocks : (q ? ch.n_tokens : 0));
  const size_t lds = (size_t)kBlockTokens * kHeadDim / 2 * sizeof(float2) + (FMT == kBf16 ? 2 : 1) * (size_t)kBlockTokens * kHeadDim * sizeof(bf16_t) +
                     (kmax ? (size_t)a.heads_per_wg * 2 * kHeadDim * pages * sizeof(bf16_t) : 0);
  const int n_kv = a.kv_wgs * a.head_groups;
  const auto kernel = rope_is_odd(r) ? append_chunk_kernel<true, FMT> : append_chunk_kernel<false, FMT>;
  hipLaunchKernelGGL(kernel, dim3(n_kv + q_wgs), dim3(kRopeT), lds, st, c, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_chunk(const CacheView& c, const ChunkView& ch, const RopeView& r, const int32_t* positions,
                               const bf16_t* q, int64_t q_stride, bf16_t* q_out, const bf16_t* k, int64_t k_stride,
                               const bf16_t* v, int64_t v_stride, bf16_t* kmax, bf16_t* kmin, void* ws, hipStream_t st) {
  return launch_append_any<kBf16>(c, nullptr, nullptr, ch, r, positions, q, q_stride, q_out, k, k_stride, v, v_stride, kmax,
                                  kmin, ws, st);
}

hipError_t launch_q_append(const QCacheView& c, const ChunkView& ch, const RopeView& r, const int32_t* positions,
                           const bf16_t* q, int64_t q_stride, bf16_t* q_out, const bf16_t* k, int64_t k_stride,
                           const bf16_t* v, int64_t v_stride, bf16_t* kmax, bf16_t* kmin, void* ws, hipStream_t st) {
  return (c.format == ROCKETKV_Q_E4M3 ? launch_append_any<ROCKETKV_Q_E4M3> : launch_append_any<ROCKETKV_Q_E2M1>)(
      c.tokens, c.k_scales, c.v_scales, ch, r, positions, q, q_stride, q_out, k, k_stride, v, v_stride, kmax, kmin, ws, st);
}

}  // namespace rkv
