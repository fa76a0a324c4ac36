// Whole caches from bf16 to codes and back.
//
// Both move a token's key and value once and compute next to nothing: memory is what bounds them.  A workgroup takes
// kConvTokens tokens of a (sequence, KV head), sixteen lanes a row of eight channels each, a page lookup per row; all its
// loads are under way before the first is used.  Values that lie by channel on the bf16 side pass through LDS, a tile of 16
// tokens at a time.
// 16 sequences of 4096 tokens of 8 heads into 8 bits, 407 MB read and written: 76 us, 5.3 TB/s (a copy of 4 GiB runs at 4.8).
// 131072 tokens in pages of 4 from 8 bits, 814 MB: 151 us, 5.4; a prompt of 32768 from 4 bits, 170 MB: 30 us, 5.7.
#include "quantise.h"

namespace rkv {

namespace {

constexpr int kConvT = 256;
constexpr int kConvTokens = 64;
constexpr int kConvRows = kConvT / 16;                 // rows a pass covers
constexpr int kConvPasses = kConvTokens / kConvRows;
constexpr int kTileRow = kHeadDim + 2;                 // of a tile in LDS: two more, so that a column's banks differ

// Tokens of both caches; what is longer than either counts as empty.
__device__ __forceinline__ int converted(const CacheView& src, const CacheView& dst, int b) {
  const int n = src.seq_lens[b];
  const int cap = min(src.pages_cap * src.page_size, dst.pages_cap * dst.page_size);
  return n < 0 || n > cap ? 0 : n;
}

// By channel, lanes 2c and 2c + 1 of a half of the workgroup hold channel c's tokens 0..7 and 8..15 of a tile.
struct TileLane {
  int channel, first;
};
__device__ __forceinline__ TileLane tile_lane() {
  return {(int)threadIdx.x / 2, (int)threadIdx.x % 2 * 8};
}

}  // namespace

struct ConvertArgs {
  CacheView bf16, codes;
  uint8_t *k_scales, *v_scales;
  int blocks;  // of kConvTokens tokens a sequence may have
};

template <int FMT, bool TOK>
__global__ __launch_bounds__(kConvT) void quantise_kernel(ConvertArgs a) {
  __shared__ bf16_t s_tile[TOK ? 1 : kAttnPage * kTileRow];
  const CacheView &src = a.bf16, &dst = a.codes;
  const int g = blockIdx.x % src.n_kv_heads, at = blockIdx.x / src.n_kv_heads, b = at / a.blocks, blk = at % a.blocks;
  const int n = converted(src, dst, b), t0 = blk * kConvTokens;
  if (blk == 0 && g == 0 && threadIdx.x == 0) dst.seq_lens[b] = n;
  if (t0 >= n) return;
  const int lane16 = threadIdx.x % 16, row = threadIdx.x / 16;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 k[kConvPasses], v[kConvPasses];
  int64_t to[kConvPasses];
#pragma unroll
  for (int u = 0; u < kConvPasses; ++u) {
    const int t = t0 + row + u * kConvRows;
    k[u] = v[u] = zero;
    to[u] = -1;
    if (TOK ? t < n : t0 + u * kAttnPage < n) {  // (by channel, a pass is a page of src, and lanes hold other tokens' values)
      const int64_t sp = phys_page(src, b, t / src.page_size);
      if (sp >= 0) {
        const int64_t off = sp * src.stride_page + g * src.stride_head;
        if (t < n) k[u] = ld16<true>(src.k_pool + off + (int64_t)(t % src.page_size) * kHeadDim + lane16 * 8);
        v[u] = ld16<true>(src.v_pool + off + (TOK ? (int64_t)(t % src.page_size) * kHeadDim + lane16 * 8
                                                  : (int64_t)tile_lane().channel * kAttnPage + tile_lane().first));
      }
      const int64_t dp = t < n ? phys_page(dst, b, t / dst.page_size) : -1;
      if (dp >= 0) to[u] = dp * dst.stride_page + g * dst.stride_head + t % dst.page_size;
    }
  }
#pragma unroll
  for (int u = 0; u < kConvPasses; ++u) {
    if (!TOK) {
      __syncthreads();  // the last tile has been read
      const TileLane tl = tile_lane();
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) s_tile[(tl.first + e) * kTileRow + tl.channel] = (bf16_t)(w[e / 2] >> (16 * (e % 2)));
      __syncthreads();
      const uint32_t* in = reinterpret_cast<const uint32_t*>(s_tile + row * kTileRow + lane16 * 8);
      v[u] = make_uint4(in[0], in[1], in[2], in[3]);
    }
    if (to[u] >= 0) {
      store_codes<FMT>(dst.k_pool, a.k_scales, to[u], lane16, quantise8<FMT>(k[u]));
      store_codes<FMT>(dst.v_pool, a.v_scales, to[u], lane16, quantise8<FMT>(v[u]));
    }
  }
}

template <int FMT, bool TOK>
__global__ __launch_bounds__(kConvT) void restore_kernel(ConvertArgs a) {
  __shared__ bf16_t s_tile[TOK ? 1 : kAttnPage * kTileRow];
  const CacheView &src = a.codes, &dst = a.bf16;
  const int g = blockIdx.x % src.n_kv_heads, at = blockIdx.x / src.n_kv_heads, b = at / a.blocks, blk = at % a.blocks;
  const int n = converted(src, dst, b), t0 = blk * kConvTokens;
  if (blk == 0 && g == 0 && threadIdx.x == 0) dst.seq_lens[b] = n;
  if (t0 >= n) return;
  const int lane16 = threadIdx.x % 16, row = threadIdx.x / 16;
  Codes8 k[kConvPasses], v[kConvPasses];
  int64_t to[kConvPasses];
#pragma unroll
  for (int u = 0; u < kConvPasses; ++u) {
    const int t = t0 + row + u * kConvRows;
    k[u] = v[u] = {make_uint2(0u, 0u), 27u};
    to[u] = -1;
    if (t < n) {
      const int64_t sp = phys_page(src, b, t / src.page_size), dp = phys_page(dst, b, t / dst.page_size);
      if (dp >= 0) to[u] = dp * dst.stride_page + g * dst.stride_head;
      if (sp >= 0) {
        const int64_t tok = sp * src.stride_page + g * src.stride_head + t % src.page_size;
        k[u] = load_codes<FMT>(src.k_pool, a.k_scales, tok, lane16);
        v[u] = load_codes<FMT>(src.v_pool, a.v_scales, tok, lane16);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kConvPasses; ++u) {
    const int t = t0 + row + u * kConvRows;
    uint4 x = restore8<FMT>(v[u].codes, v[u].scale);
    if (!TOK) {
      __syncthreads();  // the last tile has been read
      uint32_t* in = reinterpret_cast<uint32_t*>(s_tile + row * kTileRow + lane16 * 8);
      in[0] = x.x, in[1] = x.y, in[2] = x.z, in[3] = x.w;  // (zeros behind the last token)
      __syncthreads();
      const TileLane tl = tile_lane();
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = s_tile[(tl.first + 2 * e) * kTileRow + tl.channel] | (uint32_t)s_tile[(tl.first + 2 * e + 1) * kTileRow + tl.channel] << 16;
      x = make_uint4(w[0], w[1], w[2], w[3]);
      const int p = t0 / kAttnPage + u;
      const int64_t dp = p * kAttnPage < n ? phys_page(dst, b, p) : -1;
      if (dp >= 0)
        *reinterpret_cast<uint4*>(dst.v_pool + dp * dst.stride_page + g * dst.stride_head + tl.channel * kAttnPage + tl.first) = x;
    }
    if (to[u] >= 0) {
      const int64_t o = to[u] + (int64_t)(t % dst.page_size) * kHeadDim + lane16 * 8;
      *reinterpret_cast<uint4*>(dst.k_pool + o) = restore8<FMT>(k[u].codes, k[u].scale);
      if (TOK) *reinterpret_cast<uint4*>(dst.v_pool + o) = x;
    }
  }
}

namespace {
template <class Kernel>
hipError_t launch_convert(Kernel kernel, const CacheView& bf16, const QCacheView& codes, hipStream_t st) {
  ConvertArgs a = {bf16, codes.tokens, codes.k_scales, codes.v_scales, 0};
  const int64_t cap = (int64_t)bf16.pages_cap * bf16.page_size, cap2 = (int64_t)codes.tokens.pages_cap * codes.tokens.page_size;
  a.blocks = (int)(((cap < cap2 ? cap : cap2) + kConvTokens - 1) / kConvTokens);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)a.blocks * bf16.batch * bf16.n_kv_heads)), dim3(kConvT), 0, st, a);
  return hipGetLastError();
}
}  // namespace

int64_t convert_workgroups(const CacheView& bf16, const QCacheView& codes) {
  const int64_t cap = (int64_t)bf16.pages_cap * bf16.page_size, cap2 = (int64_t)codes.tokens.pages_cap * codes.tokens.page_size;
  return ((cap < cap2 ? cap : cap2) + kConvTokens - 1) / kConvTokens * bf16.batch * bf16.n_kv_heads;
}

hipError_t launch_quantise(const CacheView& src, const QCacheView& dst, hipStream_t st) {
  const bool e4m3 = dst.format == ROCKETKV_Q_E4M3;
  if (src.v_token_major) return launch_convert(e4m3 ? quantise_kernel<ROCKETKV_Q_E4M3, true> : quantise_kernel<ROCKETKV_Q_E2M1, true>, src, dst, st);
  return launch_convert(e4m3 ? quantise_kernel<ROCKETKV_Q_E4M3, false> : quantise_kernel<ROCKETKV_Q_E2M1, false>, src, dst, st);
}

hipError_t launch_restore(const QCacheView& src, const CacheView& dst, hipStream_t st) {
  const bool e4m3 = src.format == ROCKETKV_Q_E4M3;
  if (dst.v_token_major) return launch_convert(e4m3 ? restore_kernel<ROCKETKV_Q_E4M3, true> : restore_kernel<ROCKETKV_Q_E2M1, true>, dst, src, st);
  return launch_convert(e4m3 ? restore_kernel<ROCKETKV_Q_E4M3, false> : restore_kernel<ROCKETKV_Q_E2M1, false>, dst, src, st);
}

}  // namespace rkv
