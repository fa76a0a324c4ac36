// Trees of drafted tokens: who sees whom, and what stays of them in the cache.
#include "quantise.h"

namespace rkv {

namespace {

constexpr int kTreeT = 256;
constexpr int kTreeNodes = 4096;  // of a sequence whose parents are kept in LDS

}  // namespace

// A thread per row walks up its tree.  Parents stand before their children, so the words of its mask are met from the last
// to the first and each is written once.  A walk is a chain of reads, of LDS but for parents beyond kTreeNodes, and as long as
// the tree is deep: latency is all there is to it (16 trees of 32 rows 4.8 us, one of 200 5.4, a launch of next to nothing 2.5).
__global__ __launch_bounds__(kTreeT) void tree_mask_kernel(ChunkView ch, const int32_t* __restrict__ parents,
                                                           const int32_t* __restrict__ base, uint32_t* __restrict__ bits,
                                                           int words, int32_t* __restrict__ positions) {
  __shared__ int s_parent[kTreeNodes];
  const int b = blockIdx.x, row0 = chunk_first(ch, b), n = chunk_rows(ch, b);
  if ((int)blockIdx.y * kTreeT >= n) return;
  for (int i = threadIdx.x; i < min(n, kTreeNodes); i += kTreeT) s_parent[i] = parents[row0 + i];
  __syncthreads();
  const auto parent_of = [&](int i) {
    const int p = i < kTreeNodes ? s_parent[i] : parents[row0 + i];
    return p < i ? p : -1;
  };
  for (int i = blockIdx.y * kTreeT + threadIdx.x; i < n; i += gridDim.y * kTreeT) {
    uint32_t* out = bits + (int64_t)(row0 + i) * words;
    int w = i >> 5, depth = 0;
    for (int x = words - 1; x > w; --x) out[x] = 0u;
    uint32_t mine = 1u << (i & 31);
    for (int p = parent_of(i); p >= 0; p = parent_of(p)) {
      ++depth;
      for (; w > (p >> 5); --w) {
        if (w < words) out[w] = mine;
        mine = 0u;
      }
      mine |= 1u << (p & 31);
    }
    for (; w >= 0; --w) {
      if (w < words) out[w] = mine;
      mine = 0u;
    }
    if (positions) positions[row0 + i] = base[b] + depth;
  }
}

hipError_t launch_tree_mask(int batch, const ChunkView& ch, const int32_t* parents, const int32_t* base, uint32_t* bits,
                            int words, int32_t* positions, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  const int blocks = (ch.n_tokens + kTreeT - 1) / kTreeT;
  hipLaunchKernelGGL(tree_mask_kernel, dim3(batch, blocks < 32 ? blocks : 32), dim3(kTreeT), 0, st, ch, parents, base, bits,
                     words, positions);
  return hipGetLastError();
}

// Kept tokens together, a workgroup per (sequence, KV head).  A kept token never moves back, and what it goes over is no
// kept token that has not been read yet: tokens are taken in order, kMoved at a time, all read before the first is written.
// Then the summaries of the pages that changed, a thread per channel down their keys, the halves of the workgroup page about.
// Few bytes and a chain of round trips: the length, the flags, the pages, the rows, the keys of the pages that changed (5 of 32
// tokens of 16 sequences, 8 heads, bf16 6.6 us; 9 of 200 in pages of 4 in 8 bits 6.7; 7.2 and 7.9 with a page's keys requested
// one after the other).
struct KeepArgs {
  ChunkView ch;
  const uint8_t* keep;
  bf16_t *kmax, *kmin;
  uint8_t *k_scales, *v_scales;  // of a quantised cache
  uint32_t* arrived;             // per sequence at read_slot(): workgroups that have read its length
};

constexpr int kMoved = 16;  // tokens moved at a time
constexpr int kRead = 8;    // keys of a page on their way at a time

template <int FMT>
__global__ __launch_bounds__(kTreeT) void keep_kernel(CacheView c, KeepArgs a) {
  constexpr bool CODES = FMT != kBf16;
  __shared__ int s_from[kTreeT], s_count[kTreeT / kWave];
  const int g = blockIdx.x % c.n_kv_heads, b = blockIdx.x / c.n_kv_heads, tid = threadIdx.x, ps = c.page_size;
  const int row0 = chunk_first(a.ch, b), n = chunk_rows(a.ch, b);
  const int len = (int)use_late((uint32_t)c.seq_lens[b]), old = len - n;
  if (n == 0 || old < 0 || len > c.pages_cap * ps) return;
  const int lane16 = tid % 16, row = tid / 16;
  // where a token lies: its head's tile for bf16, its place among all tokens for codes; -1 if nowhere
  const auto place = [&](int t) -> int64_t {
    const int64_t pp = phys_page(c, b, t / ps);
    return pp < 0 ? -1 : pp * c.stride_page + g * c.stride_head + (CODES ? t % ps : 0);
  };
  int m = 0;  // tokens kept so far
  for (int i0 = 0; i0 < n; i0 += kTreeT) {
    const bool mine = i0 + tid < n && a.keep[row0 + i0 + tid] != 0;
    const unsigned long long all = __ballot(mine);
    __syncthreads();  // the last list has been used
    if (tid % kWave == 0) s_count[tid / kWave] = __popcll(all);
    __syncthreads();
    int before = 0, count = 0;
#pragma unroll
    for (int w = 0; w < kTreeT / kWave; ++w) {
      if (w < tid / kWave) before += s_count[w];
      count += s_count[w];
    }
    if (mine) s_from[before + __popcll(all & ((1ull << (tid % kWave)) - 1ull))] = old + i0 + tid;
    __syncthreads();
    for (int j0 = 0; j0 < count; j0 += kMoved) {
      const int moved = min(kMoved, count - j0);
      const int src = row < moved ? s_from[j0 + row] : 0, dst = old + m + j0 + row;
      const int64_t from = row < moved ? place(src) : -1, to = row < moved ? place(dst) : -1;
      if constexpr (CODES) {
        Codes8 k = {make_uint2(0u, 0u), 27u}, v = k;
        if (from >= 0) {
          k = load_codes<FMT>(c.k_pool, a.k_scales, from, lane16);
          v = load_codes<FMT>(c.v_pool, a.v_scales, from, lane16);
        }
        __syncthreads();
        if (to >= 0) {
          store_codes<FMT>(c.k_pool, a.k_scales, to, lane16, k);
          store_codes<FMT>(c.v_pool, a.v_scales, to, lane16, v);
        }
      } else {
        uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
        uint32_t x[kMoved / 2] = {};
        const int channel = tid / 2;  // by channel: a thread every other token of a channel
        if (from >= 0) {
          k = *reinterpret_cast<const uint4*>(c.k_pool + from + (src % ps) * kHeadDim + lane16 * 8);
          if (c.v_token_major) v = *reinterpret_cast<const uint4*>(c.v_pool + from + (src % ps) * kHeadDim + lane16 * 8);
        }
        if (!c.v_token_major) {
#pragma unroll
          for (int e = 0; e < kMoved / 2; ++e) {
            const int j = 2 * e + tid % 2;
            if (j < moved) {
              const int t = s_from[j0 + j];
              const int64_t at = place(t);
              if (at >= 0) x[e] = c.v_pool[at + channel * kAttnPage + t % ps];
            }
          }
        }
        __syncthreads();
        if (to >= 0) {
          *reinterpret_cast<uint4*>(c.k_pool + to + (dst % ps) * kHeadDim + lane16 * 8) = k;
          if (c.v_token_major) *reinterpret_cast<uint4*>(c.v_pool + to + (dst % ps) * kHeadDim + lane16 * 8) = v;
        }
        if (!c.v_token_major) {
#pragma unroll
          for (int e = 0; e < kMoved / 2; ++e) {
            const int j = 2 * e + tid % 2;
            if (j < moved) {
              const int t = old + m + j0 + j;
              const int64_t at = place(t);
              if (at >= 0) c.v_pool[at + channel * kAttnPage + t % ps] = (bf16_t)x[e];
            }
          }
        }
      }
      __syncthreads();
    }
    m += count;
  }
  const int end = old + m;
  if (a.kmax) {
    const int ch = tid % kHeadDim;
    const int64_t out = (((int64_t)b * c.n_kv_heads + g) * kHeadDim + ch) * c.pages_cap;
    for (int p = old / ps + tid / kHeadDim; p * ps < end; p += kTreeT / kHeadDim) {
      const int64_t at = place(p * ps);
      if (at < 0) continue;
      const int live = min(ps, end - p * ps);
      bf16_t mx = 0, mn = 0;
      for (int t0 = 0; t0 < live; t0 += kRead) {  // (the last key again in the place of those behind it)
        bf16_t x[kRead];
#pragma unroll
        for (int u = 0; u < kRead; ++u) {
          const int64_t t = min(t0 + u, live - 1);
          if constexpr (CODES) {
            const Codes8 k = load_codes<FMT>(c.k_pool, a.k_scales, at + t, ch / 8);
            const uint4 v = restore8<FMT>(k.codes, k.scale);
            const uint32_t w = ch % 8 < 4 ? (ch % 8 < 2 ? v.x : v.y) : (ch % 8 < 6 ? v.z : v.w);
            x[u] = (bf16_t)(w >> (16 * (ch % 2)));
          } else {
            x[u] = c.k_pool[at + t * kHeadDim + ch];
          }
        }
#pragma unroll
        for (int u = 0; u < kRead; ++u) {
          const float f = bf16_to_f32(x[u]);
          if (t0 + u == 0 || f > bf16_to_f32(mx)) mx = x[u];
          if (t0 + u == 0 || f < bf16_to_f32(mn)) mn = x[u];
        }
      }
      a.kmax[out + p] = mx;
      a.kmin[out + p] = mn;
    }
  }
  // The last of the sequence's workgroups to have read its length stores the new one.
  __syncthreads();
  if (tid == 0) {
    uint32_t* count = a.arrived + read_slot(c, b);
    if (__hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)c.n_kv_heads - 1) {
      clear_reads(a.arrived, read_slot(c, b));
      c.seq_lens[b] = end;
    }
  }
}

namespace {
template <int FMT>
hipError_t launch_keep_any(const CacheView& c, uint8_t* k_scales, uint8_t* v_scales, const ChunkView& ch, const uint8_t* keep,
                           bf16_t* kmax, bf16_t* kmin, void* ws, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  const KeepArgs a = {ch, keep, kmax, kmin, k_scales, v_scales,
                      reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + ROCKETKV_WS_HEADER_BYTES / 2)};
  hipLaunchKernelGGL(keep_kernel<FMT>, dim3(c.batch * c.n_kv_heads), dim3(kTreeT), 0, st, c, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_keep(const CacheView& c, const ChunkView& ch, const uint8_t* keep, bf16_t* kmax, bf16_t* kmin, void* ws,
                       hipStream_t st) {
  return launch_keep_any<kBf16>(c, nullptr, nullptr, ch, keep, kmax, kmin, ws, st);
}
hipError_t launch_q_keep(const QCacheView& c, const ChunkView& ch, const uint8_t* keep, bf16_t* kmax, bf16_t* kmin, void* ws,
                         hipStream_t st) {
  return (c.format == ROCKETKV_Q_E4M3 ? launch_keep_any<ROCKETKV_Q_E4M3> : launch_keep_any<ROCKETKV_Q_E2M1>)(
      c.tokens, c.k_scales, c.v_scales, ch, keep, kmax, kmin, ws, st);
}

}  // namespace rkv
