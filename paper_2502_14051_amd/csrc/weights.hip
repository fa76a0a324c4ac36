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
//
// What bounds it: as the attention, the matrix cores and the exponentials beside them (a product fewer, so more of the
// latter: 2048 tokens of 32 heads over 34816 keys and 8 KV heads 612 to 650 us by machine, 0.87 to 0.93 PFLOP/s); with few
// rows the one reading of the keys (one token of each of 16 sequences of 4123: 29 us, 4.8 TB/s, launch included).
#include <type_traits>

#include "attend_core.h"

namespace rkv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWeightWaves = 4, kKeyWaves = 2;  // half of them hold the same keys
constexpr int kRowStep = 128;                                           // query rows per step
constexpr int kRowStepBytes = kRowStep * kHeadDim * (int)sizeof(bf16_t);

// 16 bytes per lane, `off` bytes behind a base that is the same for the wavefront, straight to LDS
__device__ __forceinline__ void to_lds(const void* base, uint32_t off, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000),
                                           (__attribute__((address_space(3))) void*)dst, 16, (int)off, 0, 0, 0);
#endif
}

// from any address, past the caches: one token of each of 64 sequences of 8000 takes 211 us so, 218 without, 5 of 16
// sequences of up to 32000 118 and 128; 16 of 4122, called again at once, 29.8 and 29.0
__device__ __forceinline__ void to_lds_far(const void* src, unsigned char* dst) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 2);
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

constexpr int kTileKeys = kKeyWaves * 64, kWeightSlots = 512;  // keys of a workgroup; workgroups the chip holds at a time

__device__ __forceinline__ int weight_len(const CacheView& c, int b) {
  const int n = c.seq_lens[b];
  return n < 0 ? 0 : min(n, c.pages_cap * c.page_size);
}

// What a sequence's rows from `r0` on bring to the 32 keys of a wavefront, straight from memory, 32 rows at a time; the
// lane's key is `age` tokens behind the chunk's first (negative: before it), kf its channels 16 j + 8 h ..  The two halves'
// sums are to be added up.
// A row that has no log sum-exp, or does not see the key, adds exp2 of -inf.  That is NaN where its logit is NaN or +inf (or,
// in the loop of many rows, its log sum-exp is NaN).  No loop looks for it: it is the sum that shows, and is formed again
// CAREFULly, with such rows left out whatever their logit is (done so always, a step of 16 sequences took 30.5 us, 29.2 so).
template <bool CAREFUL>
__device__ __forceinline__ float sum_of_rows(const CacheView& c, const WeightArgs& a, const u32x4 (&kf)[8], float* s_lse, int g,
                                             int row0, int rows, int r0, int age, int col, int h) {
  const int G = c.group;
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  float sum = 0.f;
  for (; r0 < rows; r0 += 32) {
    const int r = min(r0 + col, rows - 1), t = r / G;
    const int64_t row = (int64_t)(row0 + t) * c.n_q_heads + (int64_t)g * G + (r - t * G);
    u32x4 qf[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) qf[j] = ld_plain<u32x4>(a.q + row * kHeadDim + h * 8 + j * 16);
    const float l = a.lse[row];
    const bool adds = l != -INFINITY && r0 + col < rows;
    if (h == 0) s_lse[col] = adds ? l * kLog2e : CAREFUL ? -INFINITY : INFINITY;
    f32x16 S;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(qf[j]), as_bf16x8(kf[j]), j == 0 ? f32x16{} : S, 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (written and read by this wavefront alone)
    const int first = max(0, age) * G - r0 - 4 * h;     // row of the block that sees the key first
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const f32x4 rl = *reinterpret_cast<const f32x4*>(&s_lse[2 * i + 4 * h]);
      float e[4];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        e[x] = 2 * i + x < first || (CAREFUL && rl[x] == -INFINITY) ? 0.f : fast_exp2(fmaf(S[i + x], sc, -rl[x]));
      part += (e[0] + e[1]) + (e[2] + e[3]);
    }
    sum += part;
    asm volatile("" ::: "memory");
  }
  return sum;
}

// The weights of those of 32 keys whose sum so far is NaN.  (Everything looked up anew, so that nothing is held for this
// through the loop in front of it.)
__device__ __forceinline__ void careful_weights(const CacheView& c, const WeightArgs& a, float* s_lse, int b, int g, int key0,
                                                float sum, int col, int h) {
  const int len = weight_len(c, b), key = key0 + col;
  const int64_t pp = key < len ? phys_page(c, b, key / c.page_size) : -1;
  const bf16_t* k = c.k_pool + (pp >= 0 ? pp * c.stride_page + (int64_t)g * c.stride_head + (int64_t)(key % c.page_size) * kHeadDim : 0) + h * 8;
  u32x4 kf[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) kf[j] = ld_plain<u32x4>(k + j * 16);
  const int n = chunk_rows(a.ch, b), old = len - n;
  const float careful = sum_of_rows<true>(c, a, kf, s_lse, g, chunk_first(a.ch, b), n * c.group, 0, key - old, col, h);
  const SwapPair sw = swap_rows32(__float_as_uint(careful));
  if (h != 0 || pp < 0 || sum == sum) return;
  const int64_t at = ((int64_t)b * c.n_kv_heads + g) * ((int64_t)c.pages_cap * c.page_size) + key;
  a.w_out[at] = (a.w_in && key < old ? a.w_in[at] : 0.f) + (__uint_as_float(sw.a) + __uint_as_float(sw.b));
}

// A wavefront holds NK blocks of 32 keys.  Two take the first 64 rows of a step, two the same keys and the other 64: a
// workgroup is done with 128 keys in half the time that four wavefronts of keys of their own take for 256, and the last
// ones of a launch leave less of the chip idle.  A unit is 32 rows; its exponentials stand beside the next unit's
// products, as in the attention, so in step `it` the rows of step it + 1 are read.
struct WeightShared {
  __align__(256) unsigned char q[2][kRowStepBytes];  // [128 rows][16 chunks], chunk x of row r at x ^ r % 16
  __align__(16) float lse[4][kRowStep];              // in the log2 domain; +inf: a row that adds nothing
  float sum[kTileKeys];
};
template <int NK>
__device__ __forceinline__ void weights_of_keys(const CacheView& c, const WeightArgs& a, WeightShared& sh, int b, int g, int key0) {
  auto& s_q = sh.q;
  auto& s_lse = sh.lse;
  auto& s_sum = sh.sum;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, h = lane / 32;
  const int kw = wave % kKeyWaves, own_rows = wave / kKeyWaves * 64;  // which 64 keys, and where in a step its rows begin
  const int G = c.group, ps = c.page_size, cap = c.pages_cap * ps;
  const int len = weight_len(c, b);
  if (key0 >= len) return;
  const int row0 = chunk_first(a.ch, b), n = chunk_rows(a.ch, b);
  const int old = len - n;  // place in the cache of the first new token (the first ones see nothing if it is negative)

  const int mine = key0 + kw * NK * 32 + col;  // this lane's first key, its next one 32 further
  bf16x8 kf[NK][8];
#pragma unroll
  for (int x = 0; x < NK; ++x) {
    const int key = mine + 32 * x;
    const int64_t pp = key < len ? phys_page(c, b, key / ps) : -1;
    const bf16_t* k = c.k_pool + (pp >= 0 ? pp * c.stride_page + (int64_t)g * c.stride_head + (int64_t)(key % ps) * kHeadDim : 0) + h * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) kf[x][j] = as_bf16x8(ld_plain<u32x4>(k + j * 16));
  }

  // rows (token, head) from the first that sees any of the workgroup's keys
  const int rows = n * G;
  const int it0 = max(0, key0 - old) * G / kRowStep, it1 = (rows + kRowStep - 1) / kRowStep;
  const uint32_t per_G = 65536u / (uint32_t)G + 1u;  // x / G == x * per_G >> 16 for x < 1024
  float lse = 0.f;
  // rows 16 wave .. of the step, and what they are normalised by; rows behind the last one repeat it
  const auto issue = [&](int it, auto to) {
    const int r0 = it * kRowStep, left = rows - r0;  // of rows in front of the first step's first row: none
    if (left <= 0) { lse = -INFINITY; return; }
    const int t0 = r0 / G, skip = r0 - t0 * G;  // the token the step begins in, and how many of its heads it leaves out
    const int64_t first = (int64_t)(row0 + t0) * c.n_q_heads + (int64_t)g * G;
    const auto place = [&](int r) {  // of a row of the step, in rows from `first`
      const uint32_t x = (uint32_t)(skip + r), t = x * per_G >> 16;
      return t * (uint32_t)c.n_q_heads + (x - t * (uint32_t)G);
    };
    // (added up here each time, rather than in eight registers of their own through the loop)
    int mine_at = wave * (kRowStep / kWeightWaves) * 256;
    asm volatile("" : "+s"(mine_at));
#pragma unroll
    for (int j = 0; j < kRowStep / kWeightWaves / 4; ++j) {
      const int r = wave * (kRowStep / kWeightWaves) + 4 * j + lane / 16;
      to_lds(a.q + first * kHeadDim, place(min(r, left - 1)) * 256u + ((lane % 16) ^ r % 16) * 16,
             s_q[decltype(to)::value] + mine_at + 4 * j * 256);
    }
    const int r = wave * kWave + lane;
    lse = r < kRowStep && r < left ? a.lse[first + place(r)] : -INFINITY;
  };
  const auto keep_lse = [&](int it) {
    if (wave < kRowStep / kWave) s_lse[it & 3][wave * kWave + lane] = lse == -INFINITY ? INFINITY : lse * kLog2e;
  };
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  const uint32_t q_at = (uint32_t)((own_rows + col) * 256 + (h ^ (col & 15)) * 16);
  const auto read_row = [&](uint32_t at, auto slot, int u, int j, bf16x8& qf) {
    qf = as_bf16x8(*reinterpret_cast<const u32x4*>(&s_q[0][0] + (at ^ (uint32_t)(32 * j)) + (decltype(slot)::value * kRowStepBytes + u * 8192)));
  };
  // Of a unit's rows the first ones may not see a key yet: key j is seen from token j - old of the chunk on.
  const int last_key = key0 + (kw + 1) * NK * 32 - 1;
  const auto mask = [&](f32x16 (&S)[NK], int r0) {
    if ((int64_t)(last_key - old) * G <= r0) return;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      const int first = max(0, mine + 32 * x - old) * G - r0 - 4 * h;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i / 4) + i % 4 < first) S[x][i] = -INFINITY;
    }
  };
  float sum[NK] = {};
  bf16x8 qf[8];
  f32x16 S[NK];
  const auto fence = []() { __builtin_amdgcn_sched_barrier(0); };
  const auto step = [&](int it, auto slot) {
    constexpr std::integral_constant<int, 1 - decltype(slot)::value> other{};
    __builtin_amdgcn_s_waitcnt(0);
    keep_lse(it + 1);
    __syncthreads();
    issue(it + 2, slot);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x16 N[NK];
      float part[NK];
      f32x4 row_lse[4];  // of rows 8 i + 4 h ..
      const uint32_t at = use_late(q_at);
      const auto read_lse = [&](int i) { row_lse[i] = *reinterpret_cast<const f32x4*>(&s_lse[it & 3][own_rows + 32 * u + 8 * i + 4 * h]); };
      read_lse(0);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        fence();
#pragma unroll
        for (int x = 0; x < NK; ++x)
          N[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[j], kf[x][j], j == 0 ? f32x16{} : N[x], 0, 0, 0);
        // (two products later the operand has been read, and its successor comes in)
        if (j >= 2) read_row(at, other, u, j - 2, qf[j - 2]);
        if (j % 2 == 0 && j < 6) read_lse(j / 2 + 1);
#pragma unroll
        for (int x = 0; x < NK; ++x) {
          const float e0 = fast_exp2(fmaf(S[x][2 * j], sc, -row_lse[j / 2][2 * j % 4]));
          const float e1 = fast_exp2(fmaf(S[x][2 * j + 1], sc, -row_lse[j / 2][2 * j % 4 + 1]));
          part[x] = j == 0 ? e0 + e1 : part[x] + (e0 + e1);
        }
      }
      fence();
      read_row(at, other, u, 6, qf[6]);
      read_row(at, other, u, 7, qf[7]);
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        sum[x] += part[x];
        S[x] = N[x];
      }
      mask(S, (it + u) * kRowStep + own_rows + 32 * (1 - u));
    }
  };
  if (it0 < it1) {
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    issue(it0, first);
    keep_lse(it0);
    issue(it0 + 1, second);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) read_row(q_at, first, 0, j, qf[j]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int x = 0; x < NK; ++x)
        S[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[j], kf[x][j], j == 0 ? f32x16{} : S[x], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) read_row(q_at, first, 1, j, qf[j]);
    mask(S, it0 * kRowStep + own_rows);
    for (int it = it0; it < it1; it += 2) {
      step(it, first);
      if (it + 1 < it1) step(it + 1, second);
    }
  }
  // (the lane counted anew: no register holds it through the loop)
  const int here = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
#pragma unroll
  for (int x = 0; x < NK; ++x) {
    const SwapPair sw = swap_rows32(__float_as_uint(sum[x]));
    sum[x] = __uint_as_float(sw.a) + __uint_as_float(sw.b);
    if (own_rows != 0 && here < 32) s_sum[(kw * NK + x) * 32 + here] = sum[x];
  }
  __syncthreads();
  if (own_rows != 0) return;
  bool again = false;
#pragma unroll
  for (int x = 0; x < NK; ++x) {
    const int at_key = (kw * NK + x) * 32 + here % 32, key = key0 + at_key;
    sum[x] += s_sum[at_key];
    const bool there = key < len && phys_page(c, b, key / ps) >= 0, odd = there && sum[x] != sum[x];
    again |= odd;
    if (here >= 32 || key >= len || odd) continue;
    const int64_t at = ((int64_t)b * c.n_kv_heads + g) * cap + key;
    const float before = a.w_in && key < old ? a.w_in[at] : 0.f;
    a.w_out[at] = there ? before + sum[x] : before;
  }
  if (!__any(again)) return;
#pragma unroll 1
  for (int x = 0; x < NK; ++x)
    careful_weights(c, a, s_lse[wave], b, g, key0 + (kw * NK + x) * 32, x == 0 ? sum[0] : sum[NK - 1], here % 32, here / 32);
}

// Tiles of 128 keys of all sequences and KV heads, the KV head running fastest: a chiplet's L2 then holds the queries of
// one head, if there are as many.  What the last round of workgroups over the chip leaves idle, if that is half of it or
// more, halves of the last tiles fill (us, without and with: 2048 tokens of 32 heads over 34816 keys and 8 KV heads, four
// and a quarter rounds, 625 and 598; 1186 tokens of 64 heads over 2242, a quarter of a round, 123 and 77).
// Other tiles took longer: 256 keys to a workgroup of four wavefronts 673, to one of eight 705, half tiles only 743.
__global__ __launch_bounds__(kWeightWaves * kWave) __attribute__((amdgpu_waves_per_eu(2)))
void weights_kernel(CacheView c, WeightArgs a) {
  __shared__ WeightShared sh;
  const int lane = threadIdx.x % kWave;
  const auto tiles_of = [&](int b) { return (weight_len(c, b) + kTileKeys - 1) / kTileKeys; };
  int tiles = 0;
  for (int b0 = 0; b0 < c.batch; b0 += kWave)
    tiles += __builtin_amdgcn_readlane((int)wave_incl_scan(b0 + lane < c.batch ? (uint32_t)tiles_of(b0 + lane) : 0u), kWave - 1);
  tiles *= c.n_kv_heads;
  const int last = tiles % kWeightSlots, halved = last <= kWeightSlots / 2 ? last : 0;
  int i = blockIdx.x, half = -1;
  if (i >= tiles - halved) {
    i -= tiles - halved;
    if (i >= 2 * halved) return;
    half = i >= halved;
    i = tiles - halved + (half ? i - halved : i);
  }
  int b, tile;
  if (!locate_tile(c.batch, i / c.n_kv_heads, tiles_of, b, tile)) return;
  const int g = i % c.n_kv_heads;
  if (half < 0) weights_of_keys<2>(c, a, sh, b, g, tile * kTileKeys);
  else weights_of_keys<1>(c, a, sh, b, g, tile * kTileKeys + half * (kTileKeys / 2));
}

// For few rows, where reading the keys once is all there is to it: a wavefront for 32 keys, nothing shared, five times the
// wavefronts.  The keys come through LDS in whole lines (a lane's own pieces of a row are 32 bytes apart from line to line:
// so 41.7 us for 16 sequences of 4123 tokens).
constexpr int kFewT = 256;
__global__ __launch_bounds__(kFewT) __attribute__((amdgpu_waves_per_eu(4)))
void weights_few_kernel(CacheView c, WeightArgs a) {
  __shared__ __align__(256) unsigned char s_k[4][32 * kHeadDim * sizeof(bf16_t)];  // chunk x of row r at x ^ r % 16
  __shared__ __align__(16) float s_lse[4][32];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, h = lane / 32;
  const int unit = blockIdx.y, b = unit / c.n_kv_heads, g = unit % c.n_kv_heads;
  const int G = c.group, ps = c.page_size, cap = c.pages_cap * ps;
  const int n_now = c.seq_lens[b], len = n_now < 0 ? 0 : min(n_now, cap);
  const int key0 = (blockIdx.x * 4 + wave) * 32, key = key0 + col;
  if (key0 >= len) return;
  const int64_t pp = key < len ? phys_page(c, b, key / ps) : -1;
  const int64_t off = pp >= 0 ? pp * c.stride_page + (int64_t)g * c.stride_head + (int64_t)(key % ps) * kHeadDim : 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int r = 4 * j + lane / 16;
    const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)(off >> 32), r) << 32 | (uint32_t)__shfl((int)off, r));
    to_lds_far(c.k_pool + at + ((lane % 16) ^ r % 16) * 8, s_k[wave] + j * 1024);
  }
  const int row0 = chunk_first(a.ch, b), n = chunk_rows(a.ch, b), old = len - n, rows = n * G;
  const float before = a.w_in && key < old && h == 0 ? a.w_in[(int64_t)unit * cap + key] : 0.f;
  u32x4 kf[8];
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (brought and read by this wavefront alone)
#pragma unroll
  for (int j = 0; j < 8; ++j) kf[j] = *reinterpret_cast<const u32x4*>(s_k[wave] + col * 256 + (((2 * j + h) ^ (col & 15)) * 16));
  const auto total_of = [&](auto careful) {
    const float sum = sum_of_rows<decltype(careful)::value>(c, a, kf, s_lse[wave], g, row0, rows, max(0, key0 - old) * G / 32 * 32,
                                                            key - old, col, h);
    const SwapPair sw = swap_rows32(__float_as_uint(sum));
    return __uint_as_float(sw.a) + __uint_as_float(sw.b);
  };
  float total = total_of(std::false_type{});
  if (__any(pp >= 0 && total != total)) {
    const float careful = total_of(std::true_type{});
    if (total != total) total = careful;
  }
  if (h == 0 && key < len) a.w_out[(int64_t)unit * cap + key] = pp >= 0 ? before + total : before;
}

int64_t weights_workgroups(const CacheView& c) {
  return ((int64_t)c.pages_cap * c.page_size + kTileKeys - 1) / kTileKeys * c.batch * c.n_kv_heads + kWeightSlots / 2;
}

hipError_t launch_weights(const CacheView& c, const ChunkView& ch, const bf16_t* q, const float* lse, const float* w_in,
                          float* w_out, hipStream_t st) {
  WeightArgs a;
  a.ch = ch;
  a.q = q;
  a.lse = lse;
  a.w_in = w_in;
  a.w_out = w_out;
  const unsigned units = (unsigned)(c.batch * c.n_kv_heads), tiles = (unsigned)((c.pages_cap * c.page_size + kTileKeys - 1) / kTileKeys);
  // By the rows of a sequence on average (us by the form for few and by the other, 32 heads over 8): 8 tokens, 32 rows, of one
  // sequence of 32000 20.6 and 34.3, of 16 of 4000 33.8 and 66.9, of 64 119.6 and 261.8; 64 rows 27.5 and 34.4, 47.8 and 67.4,
  // 162 and 262; 128 rows 40.7 and 34.4, 75.3 and 67.3, 262 and 267.  The line lies at 32, below what equal sequences ask for, as
  // the rows may as well be one sequence's: 449 tokens beside 63 single ones, all over 4000, take 274 and 281, but 2048 beside
  // 80, 105 rows a sequence, 995 and 462.
  if ((int64_t)ch.n_tokens * c.group <= 32ll * c.batch) hipLaunchKernelGGL(weights_few_kernel, dim3(tiles, units), dim3(kFewT), 0, st, c, a);
  else hipLaunchKernelGGL(weights_kernel, dim3((unsigned)weights_workgroups(c)), dim3(kWeightWaves * kWave), 0, st, c, a);
  return hipGetLastError();
}

}  // namespace rkv
