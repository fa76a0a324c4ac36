// The attention weight every cached token has received: to each key of a (sequence, KV head) the probabilities of the
// chunk's new tokens and of all query heads of the group are added,
//   w[j] += sum over heads and tokens i that see j of exp(q_i . k_j / sqrt(128) - lse_i),
// from the log sum-exp of the rows that the attention left.  The product is the first half of the attention's and is
// formed anew; what is summed is a column of it, so here the key is the product's column:
//
//   S[row][key] = Q[row][:] . K[key][:]^T     A = queries (32 rows, through LDS), B = keys, kept in registers
//
// and a lane owns one key: the 16 rows of a product are added up in its registers, one add a row, with no exchange but
// the last one with the lane 32 further.  A workgroup owns its keys over all rows, so nothing is added atomically and
// sums do not depend on the order of workgroups.
#include "attend_core.h"

namespace rkv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWeightT = 256;
constexpr int kRowStep = 64;                                       // query rows per step
constexpr int kRowStepBytes = kRowStep * kHeadDim * (int)sizeof(bf16_t);

__device__ __forceinline__ void to_lds(const bf16_t* src, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
#endif
}

}  // namespace

struct WeightArgs {
  ChunkView ch;
  const bf16_t* q;
  const float* lse;
  const float* w_in;  // null: zeros
  float* w_out;
};

// NK: blocks of 32 keys to a wavefront
template <int NK>
__global__ __launch_bounds__(kWeightT) __attribute__((amdgpu_waves_per_eu(2)))
void weights_kernel(CacheView c, WeightArgs a) {
  __shared__ __align__(16) unsigned char s_q[2][kRowStepBytes];
  __shared__ __align__(16) float s_lse[2][kRowStep];  // in the log2 domain; +inf: a row without any key
  constexpr int kKeys = 4 * 32 * NK;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, h = lane / 32;
  const int unit = blockIdx.y, b = unit / c.n_kv_heads, g = unit % c.n_kv_heads;
  const int G = c.group, ps = c.page_size, cap = c.pages_cap * ps;
  const int n_now = c.seq_lens[b], len = n_now < 0 ? 0 : min(n_now, cap);
  const int key0 = blockIdx.x * kKeys;
  if (key0 >= len) return;
  const int row0 = chunk_first(a.ch, b), n = chunk_rows(a.ch, b);
  const int old = len - n;  // place in the cache of the first new token (the first ones see nothing if it is negative)

  bf16x8 kf[NK][8];
  int key[NK];
  bool there[NK];
#pragma unroll
  for (int x = 0; x < NK; ++x) {
    key[x] = key0 + (wave * NK + x) * 32 + col;
    const int64_t pp = key[x] < len ? phys_page(c, b, key[x] / ps) : -1;
    there[x] = pp >= 0;
    const bf16_t* k = c.k_pool + (there[x] ? pp * c.stride_page + (int64_t)g * c.stride_head + (int64_t)(key[x] % ps) * kHeadDim : 0) + h * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) kf[x][j] = as_bf16x8(ld_plain<u32x4>(k + j * 16));
  }

  // rows (token, head) from the first that sees any of the workgroup's keys
  const int rows = n * G;
  const int it0 = max(0, key0 - old) * G / kRowStep, it1 = (rows + kRowStep - 1) / kRowStep;
  const auto row_at = [&](int r) {  // of a row below `rows`
    const int t = r / G;
    return (int64_t)(row0 + t) * c.n_q_heads + (int64_t)g * G + (r - t * G);
  };
  float lse = 0.f;
  const auto issue = [&](int it) {  // rows 16 wave .. of the step; chunk x of row r at x ^ r % 16
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int rr = 4 * j + lane / 16;
      const int r = min(it * kRowStep + wave * 16 + rr, rows - 1);
      to_lds(a.q + row_at(r) * kHeadDim + ((lane % 16) ^ rr) * 8, s_q[it & 1] + (wave * 16 + 4 * j) * 256);
    }
    if (wave == 0) {
      const int r = it * kRowStep + lane;
      lse = r < rows ? a.lse[row_at(r)] : -INFINITY;
    }
  };
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  float sum[NK] = {};
  if (it0 < it1) issue(it0);
  for (int it = it0; it < it1; ++it) {
    if (wave == 0) s_lse[it & 1][lane] = lse == -INFINITY ? INFINITY : lse * kLog2e;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    if (it + 1 < it1) issue(it + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r0 = it * kRowStep + 32 * u;
      if (r0 >= rows) continue;
      const unsigned char* qrow = s_q[it & 1] + (32 * u + col) * 256;
      f32x16 S[NK];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bf16x8 qf = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + (((2 * j + h) ^ (col & 15)) * 16)));
#pragma unroll
        for (int x = 0; x < NK; ++x) {
          const f32x16 zero = {};
          S[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[x][j], j == 0 ? zero : S[x], 0, 0, 0);
        }
      }
      f32x4 row_lse[4];  // of rows 8 i + 4 h ..
#pragma unroll
      for (int i = 0; i < 4; ++i) row_lse[i] = *reinterpret_cast<const f32x4*>(&s_lse[it & 1][32 * u + 8 * i + 4 * h]);
      // a row sees key j from token j - old of the chunk on
      const int first_token = r0 / G;
      const bool all = key0 + (wave + 1) * NK * 32 - 1 <= old + first_token;
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        const int first_row = max(0, key[x] - old) * G - r0;
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float e[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            e[r] = fast_exp2(fmaf(S[x][4 * i + r], sc, -row_lse[i][r]));
            if (!all && 8 * i + 4 * h + r < first_row) e[r] = 0.f;
          }
          part += (e[0] + e[1]) + (e[2] + e[3]);
        }
        sum[x] += part;
      }
    }
  }
#pragma unroll
  for (int x = 0; x < NK; ++x) {
    const SwapPair sw = swap_rows32(__float_as_uint(sum[x]));
    const float total = __uint_as_float(sw.a) + __uint_as_float(sw.b);
    if (h == 0 && key[x] < len) {
      const int64_t at = (int64_t)unit * cap + key[x];
      const float before = a.w_in && key[x] < old ? a.w_in[at] : 0.f;
      a.w_out[at] = there[x] ? before + total : before;
    }
  }
}

hipError_t launch_weights(const CacheView& c, const ChunkView& ch, const bf16_t* q, const float* lse, const float* w_in,
                          float* w_out, hipStream_t st) {
  WeightArgs a;
  a.ch = ch;
  a.q = q;
  a.lse = lse;
  a.w_in = w_in;
  a.w_out = w_out;
  const int units = c.batch * c.n_kv_heads, cap = c.pages_cap * c.page_size;
  hipLaunchKernelGGL(weights_kernel<2>, dim3((cap + 255) / 256, units), dim3(kWeightT), 0, st, c, a);
  return hipGetLastError();
}

}  // namespace rkv
