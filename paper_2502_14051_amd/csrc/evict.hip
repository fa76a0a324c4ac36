// Eviction by accumulated attention weight.  Per (sequence, KV head) of S tokens, where S exceeds keep_budget:
//   kept = the last n_recent tokens and, of the others, the keep_budget - n_recent with the largest weight
//          (ties: lower position), ascending;
// K and V rows and weights of the kept tokens move to another cache.
//
//   histogram  the weights of a slice of 16384 positions counted by bins of their ordered bits
//   collect    every slice of 4096 names the bin of the wanted rank, adds its keys in that bin to the row's list and notes
//              how many lie above it
//   select     every slice ranks the list, counts what it is preceded by, and emits its kept positions in order
//   move       64 kept tokens a workgroup
//
// Rows of up to 16384 positions need the last two only: a workgroup then holds a whole row in registers and counts and
// collects for itself.  Long rows did as well, each workgroup passing over the whole row: 27 us for 8 rows of 131072 beside 5
// for the histograms, bound by the vector instructions of that pass.
// The move is what the bytes ask for: kept rows read and written.
#include "select_core.h"
#include "vote_bins.h"

namespace rkv {

namespace {

constexpr int kEvictT = 1024;
constexpr int kEvictSlice = 4 * kEvictT;   // positions a workgroup emits at a time
constexpr int kHistSlice = 16 * kEvictT;   // positions counted into one histogram
constexpr int kEvictCand = 1024;           // keys of the wanted bin that are ranked by counting
constexpr int kEvictBatch = 8;             // pieces of four weights a thread has in flight

// Ordered bits of a weight: +0 and -0 are equal, NaN (of either sign) is above every number.
__device__ __forceinline__ uint32_t weight_key(float w) {
  return w != w ? 0xffffffffu : f32_order_key(w + 0.f);
}

// fn(position, key) for every position of the row in [from, L), by the whole workgroup; `from` and rows begin at multiples
// of 16 bytes, and rows hold a multiple of four weights
template <class Fn>
__device__ __forceinline__ void four_weights(float4 v, int j, int L, const Fn& fn) {
  const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < L) fn(j + e, weight_key(w[e]));
}
template <class Fn>
__device__ __forceinline__ void each_weight(const float* row, int from, int L, const Fn& fn) {
  for (int j0 = from + threadIdx.x * 4; j0 < L; j0 += kEvictBatch * kEvictSlice) {
    float4 v[kEvictBatch];
#pragma unroll
    for (int u = 0; u < kEvictBatch; ++u)
      if (j0 + u * kEvictSlice < L) v[u] = *reinterpret_cast<const float4*>(row + j0 + u * kEvictSlice);
#pragma unroll
    for (int u = 0; u < kEvictBatch; ++u) four_weights(v[u], j0 + u * kEvictSlice, L, fn);
  }
}

}  // namespace

struct EvictArgs {
  const float* w;       // [units][cap]
  int cap, keep, recent;
  // long rows only (hist null: short ones)
  uint16_t* hist;       // [units][hist_slices][kSelBins]
  int hist_slices;
  uint2* cand;          // [units][kEvictCand]: key, position
  uint32_t* n_cand;     // [units]
  uint32_t* above;      // [units][split]: keys above the bin in a slice
  int split;            // slices per row, a workgroup each; of kEvictSlice positions where rows are long
  int slice_len;
  int32_t* kept;        // [units][keep]
  int32_t* kept_user;   // optional copy
  float* w_out;         // optional, rows of dst_cap
  int dst_cap;
  int32_t* n_out;
};

struct EvictShared {
  uint32_t hist[kSelBins];
  uint2 cand[kEvictCand];
  uint32_t wsum[kEvictT / kWave];
  uint32_t n_cand, bin, rank, tau, need, gt, eq;
};

// The bin of rank `k` among the counts in h[], each thread's four the highest first of the ones left to it, and the rank
// within it: sh.bin, sh.rank.  Ends with a barrier.
__device__ __forceinline__ void find_rank(const uint32_t (&h)[4], uint32_t k, EvictShared& sh) {
  uint32_t above = block_excl_scan<kEvictT>(h[0] + h[1] + h[2] + h[3], sh.wsum);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (above < k && k <= above + h[i]) {
      sh.bin = (uint32_t)(kSelBins - 1 - (int)threadIdx.x * 4 - i);
      sh.rank = k - above;
    }
    above += h[i];
  }
  __syncthreads();
}
__device__ __forceinline__ void lds_counts(const EvictShared& sh, uint32_t (&h)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = sh.hist[kSelBins - 1 - threadIdx.x * 4 - i];
}
__device__ __forceinline__ void row_counts(const EvictArgs& a, int unit, int L, uint32_t (&h)[4]) {
  const int n = (L + kHistSlice - 1) / kHistSlice;
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const uint2 w = reinterpret_cast<const uint2*>(a.hist + ((int64_t)unit * a.hist_slices + s) * kSelBins)[kEvictT - 1 - threadIdx.x];
    h[0] += w.y >> 16;
    h[1] += w.y & 0xffffu;
    h[2] += w.x >> 16;
    h[3] += w.x & 0xffffu;
  }
}

__global__ __launch_bounds__(kEvictT) void evict_hist_kernel(CacheView c, EvictArgs a) {
  __shared__ uint32_t s_hist[kSelBins];
  const int unit = blockIdx.y, S = c.seq_lens[unit / c.n_kv_heads], L = S - a.recent;
  const int j0 = blockIdx.x * kHistSlice;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.n_cand[unit] = 0;
  if (S <= a.keep || S > a.cap || j0 >= L) return;
  for (int i = threadIdx.x; i < kSelBins; i += kEvictT) s_hist[i] = 0;
  __syncthreads();
  each_weight(a.w + (int64_t)unit * a.cap, j0, min(L, j0 + kHistSlice), [&](int, uint32_t key) { atomicAdd(&s_hist[vote_bin(key)], 1u); });
  __syncthreads();
  uint32_t* out = reinterpret_cast<uint32_t*>(a.hist + ((int64_t)unit * a.hist_slices + blockIdx.x) * kSelBins);
  for (int i = threadIdx.x; i < kSelBins / 2; i += kEvictT) out[i] = s_hist[2 * i] | s_hist[2 * i + 1] << 16;
}

__global__ __launch_bounds__(kEvictT) void evict_collect_kernel(CacheView c, EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x, unit = blockIdx.y, S = c.seq_lens[unit / c.n_kv_heads], L = S - a.recent;
  const int j = blockIdx.x * kEvictSlice + tid * 4;
  if (S <= a.keep || S > a.cap || (int)blockIdx.x * kEvictSlice >= L || a.keep == a.recent) return;
  const float* row = a.w + (int64_t)unit * a.cap;
  const float4 v = j < L ? *reinterpret_cast<const float4*>(row + j) : make_float4(0.f, 0.f, 0.f, 0.f);
  uint32_t h[4] = {};
  row_counts(a, unit, L, h);
  find_rank(h, (uint32_t)(a.keep - a.recent), sh);
  const KeyRange in = bin_range(sh.bin);
  uint32_t above = 0;
  four_weights(v, j, L, [&](int at, uint32_t key) {
    if (key < in.lo) return;
    if (key - in.lo > in.span) {
      ++above;
    } else {
      const uint32_t n = atomicAdd(&a.n_cand[unit], 1u);
      if (n < (uint32_t)kEvictCand) a.cand[(int64_t)unit * kEvictCand + n] = make_uint2(key, (uint32_t)at);
    }
  });
  above = wave_incl_scan(above);
  if (tid == 0) sh.gt = 0;
  __syncthreads();
  if (tid % kWave == kWave - 1) atomicAdd(&sh.gt, above);
  __syncthreads();
  if (tid == 0) a.above[(int64_t)unit * a.split + blockIdx.x] = sh.gt;
}

// SHORT: rows of at most kHistSlice positions, held in registers
template <bool SHORT>
__global__ __launch_bounds__(kEvictT) void evict_select_kernel(CacheView c, EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x, unit = blockIdx.y, b = unit / c.n_kv_heads, g = unit % c.n_kv_heads;
  const int S = c.seq_lens[b];
  int32_t* kept = a.kept + (int64_t)unit * a.keep;
  int32_t* kept2 = a.kept_user ? a.kept_user + (int64_t)unit * a.keep : nullptr;
  if (S <= a.keep || S > a.cap) {  // everything stays; a length beyond the cache counts as none, as in the other stages
    const int cnt = S > a.cap || S < 0 ? 0 : S;
    for (int i = blockIdx.x * kEvictT + tid; i < a.keep; i += gridDim.x * kEvictT) {
      const int v = i < cnt ? i : -1;
      kept[i] = v;
      if (kept2) kept2[i] = v;
    }
    if (blockIdx.x == 0 && g == 0 && tid == 0) a.n_out[b] = cnt;
    return;
  }
  const int L = S - a.recent;
  const uint32_t want = (uint32_t)(a.keep - a.recent);  // of L positions, fewer than L
  const int j_begin = blockIdx.x * a.slice_len, j_end = min(j_begin + a.slice_len, L);
  if (blockIdx.x == 0) {
    for (int i = tid; i < a.recent; i += kEvictT) {
      kept[want + i] = L + i;
      if (kept2) kept2[want + i] = L + i;
    }
    if (g == 0 && tid == 0) a.n_out[b] = a.keep;
  }
  if (j_begin >= L || want == 0) return;
  const float* row = a.w + (int64_t)unit * a.cap;
  constexpr int kHeld = SHORT ? kHistSlice / kEvictSlice : 1;
  float4 held[kHeld];  // the whole row, or the slice's first weights
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int j = (SHORT ? u * kEvictSlice : j_begin) + tid * 4;
    held[u] = j < L ? *reinterpret_cast<const float4*>(row + j) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const auto each = [&](int upto, const auto& fn) {
    if (SHORT) {
#pragma unroll
      for (int u = 0; u < kHeld; ++u) four_weights(held[u], u * kEvictSlice + tid * 4, upto, fn);
    } else {
      each_weight(row, 0, upto, fn);
    }
  };

  uint32_t h[4] = {};
  if (tid == 0) sh.n_cand = sh.gt = sh.eq = 0;
  if (SHORT) {
    for (int i = tid; i < kSelBins; i += kEvictT) sh.hist[i] = 0;
    __syncthreads();
    each(L, [&](int, uint32_t key) { atomicAdd(&sh.hist[vote_bin(key)], 1u); });
    __syncthreads();
    lds_counts(sh, h);
  } else {
    row_counts(a, unit, L, h);
  }
  find_rank(h, want, sh);
  uint32_t k = sh.rank;
  KeyRange in = bin_range(sh.bin);
  // the keys of the bin; above it, how many lie before the slice
  uint32_t gt = 0, eq = 0;
  const auto collect = [&]() {
    gt = 0;
    each(L, [&](int j, uint32_t key) {
      if (key < in.lo) return;
      if (key - in.lo > in.span) {
        gt += j < j_begin ? 1u : 0u;
      } else {
        const uint32_t at = atomicAdd(&sh.n_cand, 1u);
        if (at < (uint32_t)kEvictCand) sh.cand[at] = make_uint2(key, (uint32_t)j);
      }
    });
    __syncthreads();
    return (int)sh.n_cand;
  };
  int n_cand;
  if (SHORT) {
    n_cand = collect();
  } else {
    n_cand = (int)a.n_cand[unit];
    if (tid < min(n_cand, kEvictCand)) sh.cand[tid] = a.cand[(int64_t)unit * kEvictCand + tid];
    for (int i = tid; i < (int)blockIdx.x; i += kEvictT) gt += a.above[(int64_t)unit * a.split + i];
    __syncthreads();
  }
  // Too many to rank: the bin is divided again, each workgroup passing over its whole row.  That is rare where weights differ,
  // but 131072 zeros, or any weights of which the wanted rank is one of very many equal or below 2^-56, take 310 to 660 us a call
  // for 8 rows (37 otherwise), 16 short rows 122 to 149 (114).
  while (n_cand > kEvictCand && in.span != 0u) {
    const int shift = part_shift(in);
    __syncthreads();
    for (int i = tid; i < kSelBins; i += kEvictT) sh.hist[i] = 0;
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
    each(L, [&](int, uint32_t key) {
      if (key >= in.lo && key - in.lo <= in.span) atomicAdd(&sh.hist[(key - in.lo) >> shift], 1u);
    });
    __syncthreads();
    lds_counts(sh, h);
    find_rank(h, k, sh);
    k = sh.rank;
    in = part_range(in, sh.bin, shift);
    n_cand = collect();
  }
  uint32_t tau, need;  // the threshold, and how many keys at it are kept
  if (n_cand <= kEvictCand) {
    const uint2 own = tid < n_cand ? sh.cand[tid] : make_uint2(0u, 0xffffffffu);
    if (tid < n_cand) {
      uint32_t above = 0, upto = 0;
      for (int j = 0; j < n_cand; ++j) {
        const uint32_t other = sh.cand[j].x;
        above += other > own.x ? 1u : 0u;
        upto += other >= own.x ? 1u : 0u;
      }
      if (above < k && k <= upto) {  // equal keys write the same pair
        sh.tau = own.x;
        sh.need = k - above;
      }
    }
    __syncthreads();
    tau = sh.tau;
    need = sh.need;
    if (own.y < (uint32_t)j_begin) {
      gt += own.x > tau ? 1u : 0u;
      eq += own.x == tau ? 1u : 0u;
    }
  } else {  // one key left
    tau = in.lo;
    need = k;
    each(j_begin, [&](int, uint32_t key) { eq += key == tau ? 1u : 0u; });
  }
  gt = wave_incl_scan(gt);
  eq = wave_incl_scan(eq);
  if (tid % kWave == kWave - 1) {
    atomicAdd(&sh.gt, gt);
    atomicAdd(&sh.eq, eq);
  }
  __syncthreads();
  gt = sh.gt;
  eq = sh.eq;
  __syncthreads();

  // ordered emission: kEvictSlice positions at a time, four neighbours a thread
  for (int j0 = j_begin; j0 < j_end; j0 += kEvictSlice) {
    const int j = j0 + tid * 4;
    float4 v = held[0];
    if (SHORT) {
#pragma unroll
      for (int u = 1; u < kHeld; ++u)
        if (j0 == u * kEvictSlice) v = held[u];
    } else if (j0 != j_begin && j < j_end) {
      v = *reinterpret_cast<const float4*>(row + j);
    }
    const float w[4] = {v.x, v.y, v.z, v.w};
    uint32_t key[4], cnt = 0;  // low 16 bits: keys above the threshold, high 16 bits: keys at it
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      key[e] = weight_key(w[e]);
      if (j + e < j_end) cnt += (key[e] > tau ? 1u : 0u) + (key[e] == tau ? 0x10000u : 0u);
    }
    const uint32_t before = block_excl_scan<kEvictT>(cnt, sh.wsum);
    uint32_t mgt = gt + (before & 0xffffu), meq = eq + (before >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e >= j_end || key[e] < tau) continue;
      if (key[e] > tau || meq < need) {
        const uint32_t pos = mgt + min(meq, need);
        kept[pos] = j + e;
        if (kept2) kept2[pos] = j + e;
      }
      if (key[e] > tau) ++mgt; else ++meq;
    }
    if (j0 + kEvictSlice < j_end) {  // what this block adds to the ones after it
      if (tid == kEvictT - 1) {
        sh.gt = (before & 0xffffu) + (cnt & 0xffffu);
        sh.eq = (before >> 16) + (cnt >> 16);
      }
      __syncthreads();
      gt += sh.gt;
      eq += sh.eq;
      __syncthreads();
    }
  }
}

// 64 kept tokens to their places.  Key rows move as 256-byte rows, and so do value rows between token-major caches.
// A kept token whose page is absent counts in the destination like any other: its place is filled with zeros.
// A channel-major source tile is read whole by a wavefront, 16 bytes a lane, once for all of its kept tokens (the lines
// of its 128 channels are touched by any one of them), and the kept columns go to LDS in the order the destination wants.
template <bool SRC_TOK, bool DST_TOK>
__global__ __launch_bounds__(256) void evict_move_kernel(CacheView src, CacheView dst, EvictArgs a) {
  constexpr int kTok = 64, kColPitch = kTok + 8, kRowPitch = kHeadDim + 8;
  __shared__ int s_tok[kTok];
  __shared__ int64_t s_from[kTok];  // element offset of the token's tile, -1: absent
  __shared__ __align__(16) bf16_t s_v[SRC_TOK && DST_TOK ? 8 : DST_TOK ? kTok * kRowPitch : kHeadDim * kColPitch];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int unit = blockIdx.y, b = unit / src.n_kv_heads, g = unit % src.n_kv_heads, i0 = blockIdx.x * kTok;
  const int S = src.seq_lens[b], cnt = S > a.cap || S < 0 ? 0 : min(S, a.keep);
  if (i0 >= cnt) return;
  const int64_t shead = (int64_t)g * src.stride_head, dhead = (int64_t)g * dst.stride_head;
  if (tid < kTok) {
    const int tok = i0 + tid < cnt ? a.kept[(int64_t)unit * a.keep + i0 + tid] : -1;
    const int64_t pp = tok >= 0 ? phys_page(src, b, tok / src.page_size) : -1;
    s_tok[tid] = tok;
    s_from[tid] = pp >= 0 ? pp * src.stride_page + shead : -1;
    if (a.w_out && tok >= 0) a.w_out[(int64_t)unit * a.dst_cap + i0 + tid] = a.w[(int64_t)unit * a.cap + tok];
  }
  __syncthreads();
  const int row = tid / 16, piece = tid % 16;  // rows row, row + 16, .. of the 64; 16 bytes each
  uint4 kv[4], vv[4];
  int64_t from[4], to[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = row + 16 * u, t = i0 + i;
    from[u] = s_from[i] >= 0 ? s_from[i] + (int64_t)(s_tok[i] % src.page_size) * kHeadDim + piece * 8 : -1;
    // a channel-major destination gets whole tiles, zeros behind the end; of a token-major one the rows that exist
    const int64_t pp = (DST_TOK ? t < cnt : t / kAttnPage * kAttnPage < cnt) ? phys_page(dst, b, t / dst.page_size) : -1;
    to[u] = pp >= 0 ? pp * dst.stride_page + dhead + (int64_t)(t % dst.page_size) * kHeadDim + piece * 8 : -1;
    kv[u] = vv[u] = make_uint4(0, 0, 0, 0);
    if (from[u] >= 0) {
      kv[u] = ld16<true>(src.k_pool + from[u]);
      if (SRC_TOK) vv[u] = ld16<true>(src.v_pool + from[u]);
    }
  }
  const auto store_keys = [&]() {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (to[u] >= 0) *reinterpret_cast<uint4*>(dst.k_pool + to[u]) = kv[u];
  };
  if (SRC_TOK && DST_TOK) {
    store_keys();
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (to[u] >= 0) *reinterpret_cast<uint4*>(dst.v_pool + to[u]) = vv[u];
    return;
  }
  if (SRC_TOK) {
    store_keys();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t w[4] = {vv[u].x, vv[u].y, vv[u].z, vv[u].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) s_v[(piece * 8 + e) * kColPitch + row + 16 * u] = (bf16_t)(w[e / 2] >> (16 * (e % 2)));
    }
  } else {
    const int tok = s_tok[lane];
    const int page = s_from[lane] >= 0 ? tok / kAttnPage : -1 - lane;  // tokens without a tile are in no run
    const int left = __shfl_up(page, 1);
    unsigned long long runs = __ballot(lane == 0 || page != left);  // first tokens of the runs that share a tile
    if (s_from[lane] < 0) {  // zeros where there is nothing to read
      for (int ch = wave; ch < kHeadDim; ch += 4) s_v[DST_TOK ? lane * kRowPitch + ch : ch * kColPitch + lane] = 0;
    }
    for (int n = 0; runs != 0ull; ++n) {
      const int r0 = __ffsll(runs) - 1;
      runs &= runs - 1;
      if (n % 4 != wave) continue;
      const int r1 = runs ? __ffsll(runs) - 1 : kTok;
      const int64_t tile = s_from[r0];
      if (tile < 0) continue;
      uint4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = ld16<true>(src.v_pool + tile + (u * kWave + lane) * 8);
      for (int r = r0; r < r1; ++r) {
        const int slot = s_tok[r] % kAttnPage;
        if (slot / 8 != lane % 2) continue;  // this lane's pieces hold the other half of the tokens
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int ch = (u * kWave + lane) / 2, e = slot % 8;
          const uint32_t w = e / 2 == 0 ? x[u].x : e / 2 == 1 ? x[u].y : e / 2 == 2 ? x[u].z : x[u].w;
          s_v[DST_TOK ? r * kRowPitch + ch : ch * kColPitch + r] = (bf16_t)(w >> (16 * (e % 2)));
        }
      }
    }
    store_keys();
  }
  __syncthreads();
  if (DST_TOK) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (to[u] >= 0)
        *reinterpret_cast<uint4*>(dst.v_pool + to[u]) = *reinterpret_cast<const uint4*>(s_v + (row + 16 * u) * kRowPitch + piece * 8);
  } else {
#pragma unroll
    for (int u = 0; u < kTok / kAttnPage; ++u) {  // a destination tile at a time: channel tid / 2, tokens 8 (tid % 2) ..
      const int t = i0 + u * kAttnPage;
      const int64_t pp = t < cnt ? phys_page(dst, b, t / kAttnPage) : -1;
      if (pp >= 0)
        reinterpret_cast<uint4*>(dst.v_pool + pp * dst.stride_page + dhead)[tid] =
            *reinterpret_cast<const uint4*>(s_v + tid / 2 * kColPitch + u * kAttnPage + tid % 2 * 8);
    }
  }
}

EvictPlan plan_evict(const CacheView& src, int keep) {
  EvictPlan p;
  const size_t units = (size_t)src.batch * src.n_kv_heads;
  const int64_t cap = (int64_t)src.pages_cap * src.page_size;
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  const bool is_long = cap > kHistSlice;
  p.hist_slices = is_long ? (int)((cap + kHistSlice - 1) / kHistSlice) : 0;
  // a workgroup per slice of 4096 positions; for short rows no more workgroups than one round over the chip
  p.split = (int)((cap + kEvictSlice - 1) / kEvictSlice);
  const int most = units >= 256 ? 1 : (int)(256 / units);
  if (!is_long && p.split > most) p.split = most;
  p.slice_len = (int)(((cap + p.split - 1) / p.split + kEvictSlice - 1) / kEvictSlice * kEvictSlice);
  size_t off = ROCKETKV_WS_HEADER_BYTES;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up(bytes);
    return at;
  };
  p.kept_off = take(units * (size_t)keep * sizeof(int32_t));
  p.hist_off = take(units * (size_t)p.hist_slices * kSelBins * sizeof(uint16_t));
  p.cand_off = take(is_long ? units * kEvictCand * sizeof(uint2) : 0);
  p.n_cand_off = take(is_long ? units * sizeof(uint32_t) : 0);
  p.above_off = take(is_long ? units * (size_t)p.split * sizeof(uint32_t) : 0);
  p.total_bytes = off;
  return p;
}

hipError_t launch_evict(const CacheView& src, const float* weights, int n_recent, int keep, const CacheView& dst,
                        float* dst_weights, int32_t* kept_idx, void* ws, const EvictPlan& plan, hipStream_t st) {
  char* base = static_cast<char*>(ws);
  EvictArgs a;
  a.w = weights;
  a.cap = src.pages_cap * src.page_size;
  a.keep = keep;
  a.recent = n_recent;
  a.hist_slices = plan.hist_slices;
  a.hist = plan.hist_slices ? reinterpret_cast<uint16_t*>(base + plan.hist_off) : nullptr;
  a.cand = reinterpret_cast<uint2*>(base + plan.cand_off);
  a.n_cand = reinterpret_cast<uint32_t*>(base + plan.n_cand_off);
  a.above = reinterpret_cast<uint32_t*>(base + plan.above_off);
  a.split = plan.split;
  a.slice_len = plan.slice_len;
  a.kept = reinterpret_cast<int32_t*>(base + plan.kept_off);
  a.kept_user = kept_idx;
  a.w_out = dst_weights;
  a.dst_cap = dst.pages_cap * dst.page_size;
  a.n_out = dst.seq_lens;
  const unsigned units = (unsigned)(src.batch * src.n_kv_heads);
  const dim3 slices((unsigned)plan.split, units);
  if (a.hist) {
    hipLaunchKernelGGL(evict_hist_kernel, dim3((unsigned)plan.hist_slices, units), dim3(kEvictT), 0, st, src, a);
    hipLaunchKernelGGL(evict_collect_kernel, slices, dim3(kEvictT), 0, st, src, a);
    hipLaunchKernelGGL(evict_select_kernel<false>, slices, dim3(kEvictT), 0, st, src, a);
  } else {
    hipLaunchKernelGGL(evict_select_kernel<true>, slices, dim3(kEvictT), 0, st, src, a);
  }
  const dim3 grid((unsigned)((keep + 63) / 64), units), block(256);
  if (src.v_token_major) {
    if (dst.v_token_major) hipLaunchKernelGGL((evict_move_kernel<true, true>), grid, block, 0, st, src, dst, a);
    else hipLaunchKernelGGL((evict_move_kernel<true, false>), grid, block, 0, st, src, dst, a);
  } else {
    if (dst.v_token_major) hipLaunchKernelGGL((evict_move_kernel<false, true>), grid, block, 0, st, src, dst, a);
    else hipLaunchKernelGGL((evict_move_kernel<false, false>), grid, block, 0, st, src, dst, a);
  }
  return hipGetLastError();
}

}  // namespace rkv
