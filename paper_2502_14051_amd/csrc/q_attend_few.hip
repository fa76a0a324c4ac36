// Attention of few rows over a quantised cache: decode steps and short drafts, where the keys are read once and what
// counts is how fast they come.
//
// Rows of a (sequence, KV head) are its new tokens times the group's query heads, NB tiles of 16.  Every wavefront walks
// keys of its own, 32 at a time, with the running maximum m and sum l of each row, and the wavefronts' results are joined
// through LDS, then those of the workgroups that share a tile's keys, by the one of them that is done last:
//
//   S^T[key][row]    = K[key][:] . Q[row][:]              A = 16 keys, B = 16 rows
//   O^T[chan][row]  += V^T[chan][key] . P^T[key][row]     A = 16 channels, B = exp2(S c - m) of 32 keys
//
// Lane (i, kg) of a wavefront, i = lane % 16, kg = lane / 16, takes 32 channels of key row i, 16 bytes of codes at a time that
// are next to its neighbours': channels 32 kg .. (E2M1), or 16 kg .. and 64 + 16 kg .. (E4M3).  The queries are held in the
// same order.  The rows of the two tiles of 16 keys are keys
// 8 (i / 4) + 4 x + i % 4, x = 0, 1, so that the logits it gets are those of keys 8 kg .. 8 kg + 7 of row i, which packed to
// bf16 are the second product's operand as they stand.  Keys thus go from memory to registers and, widened, into the matrix
// cores; values have to be turned and pass through 8 KiB of LDS of the wavefront's own, without a barrier.
#include "chunk_attend_core.h"
#include "few_division.h"

namespace rkv {

namespace {

constexpr int few_waves(int tiles) { return tiles == 1 ? 16 : 8; }  // as many as registers allow
constexpr int kUnit = 32;                                       // keys a wavefront takes at a time
constexpr int kUnitBytes = kUnit * kHeadDim * (int)sizeof(bf16_t);  // values of a unit, a tile's outputs

typedef float f4 __attribute__((ext_vector_type(4)));

// All bits of those of a pair of bf16 values that are no finite numbers.
__device__ __forceinline__ uint32_t no_numbers(uint32_t pair) {
  return ((pair & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((pair & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Partial results handed from one workgroup to another, four at a time, past the caches that do not see each other (the
// scope that atomics have for the whole device).
[[maybe_unused]] constexpr int kDeviceScope = 16;
__device__ __forceinline__ void st_agent4(float* base, uint32_t at, f4 v) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), __builtin_amdgcn_make_buffer_rsrc(base, 0, -1, 0x00020000), (int)(at * 4u), 0, kDeviceScope);
#endif
}
__device__ __forceinline__ f4 ld_agent4(float* base, uint32_t at) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc(base, 0, -1, 0x00020000), (int)(at * 4u), 0, kDeviceScope));
#else
  return f4{};
#endif
}

// Where workgroup `at` of a KV head works, found by one wavefront.
template <View VIEW>
__device__ __forceinline__ bool few_place(const CacheView& c, const ChunkAttendArgs& a, int at, ChunkPlace& p, ChunkSeq& s) {
  const int lane = threadIdx.x % kWave;
  const ChunkSeq own = chunk_seq_of_lane<VIEW>(c, a);
  const auto total = [](int x) { return __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)x), kWave - 1); };
  const auto tiles_of = [&](const ChunkSeq& s) { return VIEW == kListed ? 1 : chunk_ceil(s.n, a.tile_tokens); };
  const auto each = [&](const auto& fn) {  // of the tiles and units of every sequence
    for (int b0 = 0; b0 < c.batch; b0 += kWave) {
      int t = 0, units = 0;
      if (b0 + lane < c.batch) {
        const ChunkSeq s = b0 == 0 ? own : chunk_seq<VIEW>(c, a, b0 + lane);
        t = tiles_of(s);
        units = t ? chunk_ceil(s.len, 32) : 0;
      }
      fn(t, units);
    }
  };
  float share = 0.f;
  if (a.partial) {
    int tiles = 0;
    float work = 0.f;
    each([&](int t, int units) {
      tiles += total(t) * c.n_kv_heads;
      // (a coarser count keeps the sums in range where sequences are long: 2^16 units are 2^21 tokens)
      work += (float)total(min(t, a.most) * min(units, 1 << 16)) * (float)c.n_kv_heads;
    });
    share = few_share(work, tiles, a.most, [&](float x) {
      int n = 0;
      each([&](int t, int units) { n += total(t * few_parts(units, x)); });
      return n * c.n_kv_heads;
    });
  }
  int idx;
  if (!locate_tile(c.batch, at, [&](int i) {
        const ChunkSeq s = i < kWave ? own : chunk_seq<VIEW>(c, a, i);
        return tiles_of(s) * few_parts(chunk_ceil(s.len, 32), share);
      }, p.b, idx))
    return false;
  if (p.b < kWave) s = {__builtin_amdgcn_readlane(own.row, p.b), __builtin_amdgcn_readlane(own.n, p.b), __builtin_amdgcn_readlane(own.len, p.b)};
  else s = chunk_seq<VIEW>(c, a, p.b);
  p.parts = few_parts(chunk_ceil(s.len, 32), share);
  p.next = tiles_of(s);
  p.part = idx / p.next;
  p.tile = p.next - 1 - idx % p.next;
  p.first = at - p.part * p.next;
  return true;
}

}  // namespace

template <Source SRC, View VIEW, int NB>
__global__ __launch_bounds__(few_waves(NB) * kWave) __attribute__((amdgpu_waves_per_eu(NB == 1 ? 4 : 2)))
void few_attend_kernel(CacheView c, ChunkAttendArgs a, uint32_t* counters) {
  constexpr int kRows = 16 * NB, kWaves = few_waves(NB);
  constexpr int kRowBytes = SRC == kE4M3 ? kHeadDim : kHeadDim / 2;
  constexpr int kKeyLoads = SRC == kE4M3 ? 2 : 1;  // of 16 bytes, a lane's 32 codes of a key
  typedef typename Codes16<SRC>::Raw Raw;
  extern __shared__ __align__(256) unsigned char s_tiles[];  // [wavefront] a unit's values; later a row tile's outputs
  __shared__ float s_stats[kWaves][kRows][3];  // later [half a wavefront] of those that join parts
  __shared__ u32x4 s_q[NB * 4 * kWave];
  __shared__ int s_last;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i16 = lane % 16, kg = lane / 16;
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads;
  // Lists are all of one length, which the host divides; sequences are divided here, by one wavefront for all.
  ChunkPlace pl;
  ChunkSeq s;
  if (VIEW == kListed && a.pages) {
    const int b = at % c.batch;
    pl = {b, 0, at / c.batch, a.list_parts, b, c.batch};
    s = {b, 1, a.row_len * c.page_size};
  } else {
    __shared__ ChunkPlace s_place;
    __shared__ ChunkSeq s_seq;
    if (wave == 0) {
      if (!few_place<VIEW>(c, a, at, pl, s)) pl.parts = 0;
      if (lane == 0) s_place = pl, s_seq = s;
    }
    __syncthreads();
    const auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    pl = {same(s_place.b), same(s_place.tile), same(s_place.part), same(s_place.parts), same(s_place.first), same(s_place.next)};
    s = {same(s_seq.row), same(s_seq.n), same(s_seq.len)};
    if (pl.parts == 0) return;
  }
  if (pl.parts > 1 && (int)blockIdx.x >= a.most) return;  // (`starts` that overlap)
  const int G = c.group, ps = c.page_size;
  const int t0 = pl.tile * a.tile_tokens, nt = min(a.tile_tokens, s.n - t0);
  const int rows = nt * G;
  const int old = s.len - s.n, pos0 = old + t0;

  // the part's units
  const int units = chunk_ceil(max(0, VIEW == kMasked ? s.len : min(s.len, pos0 + nt)), kUnit);
  const int u0 = (int)((int64_t)units * pl.part / pl.parts), u1 = (int)((int64_t)units * (pl.part + 1) / pl.parts);

  const auto packed_row = [&](int r) {  // (token, head) of the packed tensors
    const int t = r / G;
    return (int64_t)(s.row + t0 + t) * c.n_q_heads + (int64_t)g * G + (r - t * G);
  };
  int last[NB];  // the last key each row sees
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = nb * 16 + i16;
    last[nb] = r < rows ? pos0 + r / G : -1;
  }
  // The queries as every wavefront's lanes read them (from LDS, unit after unit: registers are what there is little of).
  for (int x = threadIdx.x; x < NB * 4 * kWave; x += kWaves * kWave) {
    const int ln = x % kWave, j = x / kWave % 4, r = x / (4 * kWave) * 16 + ln % 16;
    const int channel = SRC == kE4M3 ? j / 2 * 64 + ln / 16 * 16 + j % 2 * 8 : ln / 16 * 32 + 8 * j;
    u32x4 v = *reinterpret_cast<const u32x4*>(a.q + packed_row(min(r, rows - 1)) * kHeadDim + channel);
    if (r >= rows) v = (u32x4){0u, 0u, 0u, 0u};
    s_q[x] = v;
  }
  const int sees_first = VIEW == kMasked ? old - 1 : pos0;  // the last key that all rows see

  // Where the tokens of a unit lie, lane i of the first 32 token i, looked up a unit ahead (and a list's pages two).
  struct Found {
    int raw, slot;
  };
  const int list_len = VIEW == kListed ? min(max(c.seq_lens[pl.b], 0), c.pages_cap * ps) : 0;
  // (a lane's places are derived anew at each use: held over the loop they would take the registers that are left)
  const auto fresh = [&]() { return use_late((uint32_t)lane); };
  const auto list_entry = [&](int u) {
    const uint32_t t = (uint32_t)(u * kUnit) + fresh() % kUnit, p = t / (uint32_t)ps;
    const int32_t* row = a.pages + ((int64_t)pl.b * c.n_kv_heads + g) * a.row_len;
    return Found{u >= u1 || (int)t >= s.len ? -1 : a.pages ? row[p] : (int)p, (int)(t - p * ps)};
  };
  const auto find = [&](int u, Found e) {
    if (VIEW == kListed) {
      const bool there = e.raw >= 0 && e.raw < c.pages_cap && e.raw * ps + e.slot < list_len;
      return Found{there ? phys_page_request(c, pl.b, e.raw) : -1, e.slot};
    }
    const uint32_t t = (uint32_t)(u * kUnit) + fresh() % kUnit, p = t / (uint32_t)ps;
    return Found{u < u1 && (int)t < s.len ? phys_page_request(c, pl.b, (int)p) : -1, (int)(t - p * ps)};
  };

  u32x4 k_raw[2][kKeyLoads];
  uint32_t k_scale[2], v_scale[4];
  Raw v_raw[4];
  const auto request = [&](Found f) {  // returns a bit per token that exists
    const bool there = f.raw >= 0 && (int64_t)f.raw < c.n_phys_pages;
    const uint32_t tok = there ? (uint32_t)(f.raw * c.stride_page + g * c.stride_head + f.slot) : 0u;
    const uint32_t valid = (uint32_t)__ballot(there);
    const uint8_t* vs = reinterpret_cast<const uint8_t*>(a.v_scales);
    const uint32_t ln = fresh();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint64_t r = (uint32_t)__shfl((int)tok, (int)(8 * (ln % 16 / 4) + 4 * x + ln % 4));
      const u32x4* src = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(c.k_pool) + r * kRowBytes) + ln / 16;
#pragma unroll
      for (int p = 0; p < kKeyLoads; ++p) k_raw[x][p] = src[4 * p];
      k_scale[x] = a.k_scales[r];
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint64_t r = (uint32_t)__shfl((int)tok, (int)(8 * p + ln / 8));
      v_raw[p] = __builtin_nontemporal_load(reinterpret_cast<const Raw*>(reinterpret_cast<const char*>(c.v_pool) + r * kRowBytes) + ln % 8);
      v_scale[p] = vs[r * 4 + ln % 8 / 2];
    }
    return valid;
  };

  f4 O[NB][8];
  float m[NB], l[NB], lr[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = kNegBig, l[nb] = lr[nb] = 0.f;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) O[nb][cb] = (f4){0.f, 0.f, 0.f, 0.f};
  }
  const float sc = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)
  unsigned char* mine = s_tiles + wave * kUnitBytes;

  // Keys of row `nb * 16 + i16` among the 32 from key0 on, a bit each.
  const auto seen_bits = [&](int key0, int nb) -> uint32_t {
    if (last[nb] < 0) return 0u;
    if (VIEW != kMasked) {
      const int n = last[nb] - key0 + 1;
      return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    }
    const int j = key0 - old;
    if (j <= -32) return ~0u;
    const uint32_t* tile = a.mask + (int64_t)(s.row + t0) * a.mask_words;
    const int w = j >> 5, place = (int)((nb * 16 + fresh() % 16) / (uint32_t)G) * a.mask_words + w;
    const uint32_t lo = w < 0 ? ~0u : w < a.mask_words ? tile[place] : 0u, hi = w + 1 < a.mask_words ? tile[place + 1] : 0u;
    return (uint32_t)(((uint64_t)hi << 32 | lo) >> (j & 31));
  };

  // values by channel: lane i of 16 names piece i % 4 of block row i / 4, see lds_columns
  // Its address: chunk 2 cb + i % 4 / 2 of a row turned by 4 (i / 4), so blocks 2x and 2x + 1 lie 32 bytes apart, and x turns two bits.
  const auto values_at = [&]() {
    const uint32_t ln = fresh();
    return (uint32_t)(wave * kUnitBytes) + (8 * (ln / 16) + ln % 16 / 4) * 256 + (ln % 4 / 2) * 16 + (ln % 16 / 4) * 64 + ln % 2 * 8;
  };
  const auto values = [&](uint32_t at, int cb) {
    u32x2 w[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) w[z] = lds_columns(s_tiles + ((at ^ (uint32_t)(cb / 2 * 64)) + (cb % 2 * 32 + z * 1024)));
    return as_bf16x8((u32x4){w[0].x, w[0].y, w[1].x, w[1].y});
  };
  int odd_from = -1;  // the first unit with a value that is no number among keys that not all rows see
  int u = u0 + wave;
  Found entry = {-1, 0}, found = {-1, 0};
  uint32_t valid = 0;
  if (u < u1) {
    if (VIEW == kListed) {
      const Found e0 = list_entry(u), e1 = list_entry(u + kWaves);
      entry = list_entry(u + 2 * kWaves);
      const Found f = find(u, e0);
      found = find(u + kWaves, e1);
      valid = request(f);
    } else {
      const Found f = find(u, entry);
      found = find(u + kWaves, entry);
      valid = request(f);
    }
  }
  __syncthreads();
  for (; u < u1; u += kWaves) {
    const int key0 = u * kUnit;
    const uint32_t there = valid;
    // values to LDS: chunk x of row r at x ^ 4 (r % 4)
    const bool partly = there != ~0u || key0 + kUnit - 1 > sees_first, apart = VIEW != kListed && partly && rows > G;
    bool odd = false;
    {
      const uint32_t ln = fresh();
      // (rows 8 further turn alike)
      const uint32_t to = (uint32_t)(wave * kUnitBytes) + ln / 8 * 256 + (((2 * (ln % 8)) ^ (4 * (ln / 8 % 4))) * 16);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        u32x4 lo, hi;
        widen16(v_raw[p], __uint_as_float(v_scale[p] << 23), lo, hi);
        if (partly) {
          if (!(there >> (8 * p + ln / 8) & 1u)) lo = hi = (u32x4){0u, 0u, 0u, 0u};  // (0 x NaN is not 0)
          if (apart) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = no_numbers(lo[e]), y = no_numbers(hi[e]);
              lo[e] &= ~x, hi[e] &= ~y;
              odd |= (x | y) != 0u;
            }
          }
        }
        *reinterpret_cast<u32x4*>(s_tiles + (to + p * 2048)) = lo;
        *reinterpret_cast<u32x4*>(s_tiles + ((to ^ 16u) + p * 2048)) = hi;
      }
      if (apart && odd_from < 0 && __any(odd)) odd_from = u;
    }
    f4 S[NB][2];
    const u32x4* queries = s_q + fresh();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      u32x4 kf[4];
      const uint32_t scales = k_scale[x] >> (SRC == kE4M3 ? fresh() / 32 * 8 : fresh() / 16 * 8);  // its first block's below
      const float by = __uint_as_float((scales & 0xffu) << 23);
      if constexpr (SRC == kE4M3) {
        widen16(k_raw[x][0], by, kf[0], kf[1]);
        widen16(k_raw[x][1], __uint_as_float((scales >> 16 & 0xffu) << 23), kf[2], kf[3]);
      } else {
        widen16((u32x2){k_raw[x][0].x, k_raw[x][0].y}, by, kf[0], kf[1]);
        widen16((u32x2){k_raw[x][0].z, k_raw[x][0].w}, by, kf[2], kf[3]);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          S[nb][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[j]), as_bf16x8(queries[(nb * 4 + j) * kWave]), j == 0 ? (f4){0.f, 0.f, 0.f, 0.f} : S[nb][x], 0, 0, 0);
    }
    // what the next unit brings, while this one is worked on
    if (u + kWaves < u1) {
      valid = request(found);
      found = find(u + 2 * kWaves, entry);
      if (VIEW == kListed) entry = list_entry(u + 3 * kWaves);
    }
    u32x4 pf[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (partly || NB * 16 > rows) {
        const uint32_t ok = (there & seen_bits(key0, nb)) >> (8 * kg);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(ok >> e & 1u)) S[nb][e / 4][e % 4] = -INFINITY;
      }
      float p[8], sum;
      const auto exponentials = [&]() {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = fast_exp2(fmaf(S[nb][e / 4][e % 4], sc, -m[nb]));
        sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      };
      exponentials();
      // (the maximum is followed only where sums relative to the old one outgrow 2^16, the first keys' always)
      if (__any(!(sum <= kSumLimit))) {
        float mx = S[nb][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, S[nb][e / 4][e % 4]);
        mx = rows_max_f32(mx) * sc;
        const float mn = mx > m[nb] + kLazy ? mx : m[nb], alpha = fast_exp2(m[nb] - mn);
        m[nb] = mn;
        l[nb] *= alpha;
        lr[nb] *= alpha;
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) O[nb][cb] *= alpha;
        exponentials();
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) pf[nb][e] = pack_bf16x2(p[2 * e], p[2 * e + 1]);
      float rounded = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) rounded = add_rounded(pf[nb][e], rounded);
      l[nb] += sum;
      lr[nb] += rounded;
    }
    const uint32_t values_from = values_at();
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) {
      const bf16x8 vf = values(values_from, cb);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) O[nb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, as_bf16x8(pf[nb]), O[nb][cb], 0, 0, 0);
    }
  }

  // Values that are no numbers, of keys that not all rows see: where a row sees any in a channel, which a product of zeros and
  // ones says, its result is none either.
  if (VIEW != kListed && odd_from >= 0) {
#pragma unroll 1
    for (u = odd_from; u < u1; u += kWaves) {
      const int key0 = u * kUnit;
      const uint32_t ln = fresh();
      const Found f = find(u, entry);
      const bool here = f.raw >= 0 && (int64_t)f.raw < c.n_phys_pages;
      const uint32_t tok = here ? (uint32_t)(f.raw * c.stride_page + g * c.stride_head + f.slot) : 0u;
      const uint32_t there = (uint32_t)__ballot(here);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint32_t r = 8 * p + ln / 8;
        const uint64_t row = (uint32_t)__shfl((int)tok, (int)r);
        u32x4 lo, hi;
        widen16(*(reinterpret_cast<const Raw*>(reinterpret_cast<const char*>(c.v_pool) + row * kRowBytes) + ln % 8),
                __uint_as_float((uint32_t)reinterpret_cast<const uint8_t*>(a.v_scales)[row * 4 + ln % 8 / 2] << 23), lo, hi);
        const uint32_t ones = there >> r & 1u ? 0x3f803f80u : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) lo[e] = no_numbers(lo[e]) & ones, hi[e] = no_numbers(hi[e]) & ones;
        const uint32_t x = (2 * (ln % 8)) ^ (4 * (r & 3));
        *reinterpret_cast<u32x4*>(mine + r * 256 + x * 16) = lo;
        *reinterpret_cast<u32x4*>(mine + r * 256 + (x ^ 1) * 16) = hi;
      }
      u32x4 seen[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t ok = (there & seen_bits(key0, nb)) >> (8 * kg);
#pragma unroll
        for (int e = 0; e < 4; ++e) seen[nb][e] = (ok >> (2 * e) & 1u ? 0x3f80u : 0u) | (ok >> (2 * e + 1) & 1u ? 0x3f800000u : 0u);
      }
      const uint32_t values_from = values_at();
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) {
        const bf16x8 vf = values(values_from, cb);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f4 any = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, as_bf16x8(seen[nb]), (f4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) O[nb][cb][e] = any[e] > 0.f ? __uint_as_float(0x7fc00000u) : O[nb][cb][e];
        }
      }
    }
  }

  // The wavefronts' results, a row tile at a time: four channels q of row i at place q ^ i, so that rows differ in banks.
  const uint32_t part_row = (uint32_t)(at * c.n_kv_heads + g) * kRows;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb > 0) __syncthreads();
    const float ls = rows_sum_f32(l[nb]), lrs = rows_sum_f32(lr[nb]);
    if (kg == 0) {
      float* st = s_stats[wave][nb * 16 + i16];
      st[0] = m[nb], st[1] = ls, st[2] = lrs;
    }
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) *reinterpret_cast<f4*>(mine + i16 * 512 + ((4 * cb + kg) ^ i16) * 16) = O[nb][cb];
    __syncthreads();
    for (int idx = threadIdx.x; idx < min(rows - nb * 16, 16) * 32; idx += kWaves * kWave) {
      const int i = idx / 32, q = idx % 32, r = nb * 16 + i;
      float M = kNegBig;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_stats[w][r][0]);
      float sum = 0.f, rounded = 0.f;
      f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = fast_exp2(s_stats[w][r][0] - M);
        sum = fmaf(s_stats[w][r][1], f, sum);
        rounded = fmaf(s_stats[w][r][2], f, rounded);
        const f4 x = *reinterpret_cast<const f4*>(s_tiles + w * kUnitBytes + i * 512 + (q ^ i) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], f, o[e]);
      }
      if (pl.parts == 1) {
        const float inv = sum == 0.f ? 0.f : 1.f / rounded;  // (a sum that is NaN stays one: only 0 is no key at all)
        const int64_t row = packed_row(r);
        *reinterpret_cast<u32x2*>(a.out + row * kHeadDim + 4 * q) = (u32x2){pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        if (a.out_lse && q == 0) a.out_lse[row] = sum == 0.f ? -INFINITY : (M + __log2f(sum)) * kLn2;
      } else {
        const float fit = sum == 0.f ? 0.f : sum / rounded;  // (so that the merge needs one sum)
        st_agent4(a.partial, (part_row + r) * kHeadDim + 4 * q, o * fit);
        if (q == 0) {
          float* st = reinterpret_cast<float*>(a.part_stats + part_row + r);
          st_agent(st, M);
          st_agent(st + 1, sum);
        }
      }
    }
  }
  if (pl.parts == 1) return;

  // Whoever of the tile's workgroups is done last joins their results.  (See the hand-off of data between workgroups.)
  drain_stores();
  __syncthreads();
  uint32_t* counter = counters + pl.first * c.n_kv_heads + g;
  if (threadIdx.x == 0)
    s_last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)pl.parts - 1;
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // 32 lanes a row, as many threads beside each other on its parts as there are to spare
  constexpr int kSlots = kWaves * 2;
  const int share = max(1, kSlots / rows), slot = threadIdx.x / 32, q = threadIdx.x % 32;
  const uint32_t row0 = (uint32_t)(pl.first * c.n_kv_heads + g) * kRows, next = (uint32_t)(pl.next * c.n_kv_heads) * kRows;
  for (int r0 = 0; r0 < rows; r0 += kSlots / share) {
    const int r = r0 + slot / share, first = slot % share;
    const bool works = r < rows && slot / share < kSlots / share;
    float (*s_join)[3] = s_stats[0];
    float M = kNegBig, sum = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    if (works)
      for (int p0 = first; p0 < pl.parts; p0 += 4 * share) {
        f4 v[4];
        float ms[4], ss[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {  // (absent ones weigh nothing, and read the first)
          const bool ok = p0 + x * share < pl.parts;
          const uint32_t pr = row0 + (uint32_t)(ok ? p0 + x * share : p0) * next + r;
          const float* st = reinterpret_cast<const float*>(a.part_stats + pr);
          ms[x] = ld_agent(st), ss[x] = ld_agent(st + 1);
          v[x] = ld_agent4(a.partial, pr * kHeadDim + 4 * q);
          if (!ok) ms[x] = kNegBig, ss[x] = 0.f, v[x] = (f4){0.f, 0.f, 0.f, 0.f};
        }
        float Mn = M;
#pragma unroll
        for (int x = 0; x < 4; ++x) Mn = fmaxf(Mn, ms[x]);
        const float fo = fast_exp2(M - Mn);
        sum *= fo;
        o *= fo;
        M = Mn;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float f = fast_exp2(ms[x] - M);
          sum = fmaf(ss[x], f, sum);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(v[x][e], f, o[e]);
        }
      }
    if (share > 1) {
      __syncthreads();
      if (q == 0) s_join[slot][0] = M, s_join[slot][1] = sum;
      *reinterpret_cast<f4*>(s_tiles + slot * 512 + q * 16) = o;
      __syncthreads();
      if (first == 0 && works) {
        float Mn = M;
        for (int x = 1; x < share; ++x) Mn = fmaxf(Mn, s_join[slot + x][0]);
        float f = fast_exp2(M - Mn);
        sum *= f;
        o *= f;
        for (int x = 1; x < share; ++x) {
          f = fast_exp2(s_join[slot + x][0] - Mn);
          sum = fmaf(s_join[slot + x][1], f, sum);
          const f4 v = *reinterpret_cast<const f4*>(s_tiles + (slot + x) * 512 + q * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], f, o[e]);
        }
        M = Mn;
      }
    }
    if (works && first == 0) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int64_t row = packed_row(r);
      *reinterpret_cast<u32x2*>(a.out + row * kHeadDim + 4 * q) = (u32x2){pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
      if (a.out_lse && q == 0) a.out_lse[row] = sum == 0.f ? -INFINITY : (M + __log2f(sum)) * kLn2;
    }
  }
}

void plan_few(const CacheView& c, int n_tokens, int tiles, ChunkPlan& p) {
  p.far = p.stream = false;
  p.tile_rows = 16 * tiles;
  p.tile_tokens = p.tile_rows / c.group;
  p.slots = 256 * (16 / few_waves(tiles));
  p.most = p.slots;
  int64_t most_tiles = (int64_t)n_tokens / p.tile_tokens + c.batch;
  if (most_tiles > n_tokens) most_tiles = n_tokens;
  most_tiles *= c.n_kv_heads;
  const int64_t at_least = ((int64_t)n_tokens + p.tile_tokens - 1) / p.tile_tokens * c.n_kv_heads;
  // (where no sequence can be long enough to be cut, only the workgroups of tiles are launched)
  p.cuts = at_least < p.most && (int64_t)c.pages_cap * c.page_size > 2 * kFewRound * kUnit;
  p.workgroups = p.cuts && most_tiles < p.most ? p.most : most_tiles;
}

void plan_few_listed(const CacheView& c, int row_len, ChunkPlan& p) {
  plan_few(c, c.batch, 1, p);
  const int units = (int)(((int64_t)row_len * c.page_size + kUnit - 1) / kUnit), lists = c.batch * c.n_kv_heads;
  p.list_parts = few_parts(units, few_share((float)lists * (float)units, lists, p.slots, [&](float x) { return lists * few_parts(units, x); }));
  p.cuts = p.list_parts > 1;
  p.workgroups = (int64_t)lists * p.list_parts;
}

template <View VIEW>
hipError_t launch_few(const QCacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, uint32_t* counters, hipStream_t st) {
  const int tiles = plan.tile_rows / 16;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.workgroups), dim3(few_waves(tiles) * kWave), few_waves(tiles) * kUnitBytes, st, c.tokens, a, counters);
    return hipGetLastError();
  };
  const bool e4m3 = c.format == ROCKETKV_Q_E4M3;
  if constexpr (VIEW != kListed)
    if (plan.tile_rows == 32) return e4m3 ? launch(few_attend_kernel<kE4M3, VIEW, 2>) : launch(few_attend_kernel<kE2M1, VIEW, 2>);
  return e4m3 ? launch(few_attend_kernel<kE4M3, VIEW, 1>) : launch(few_attend_kernel<kE2M1, VIEW, 1>);
}

hipError_t launch_few_attend(const QCacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, bool listed, uint32_t* counters,
                             hipStream_t st) {
  if (listed) return launch_few<kListed>(c, a, plan, counters, st);
  return a.mask ? launch_few<kMasked>(c, a, plan, counters, st) : launch_few<kCausal>(c, a, plan, counters, st);
}

}  // namespace rkv
