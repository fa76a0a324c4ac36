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
// same order.  The rows of the two tiles of 16 keys are keys 8 (i / 4) + 4 x + i % 4, x = 0, 1, so that the logits it gets are
// those of keys 8 kg .. 8 kg + 7 of row i, which packed to bf16 are the second product's operand as they stand.  Keys thus go
// from memory to registers and, widened, into the matrix cores; values have to be turned and pass through 8 KiB of LDS of the
// wavefront's own, without a barrier.
//
// What bounds it: memory, once a launch has filled the chip.  A key and its value are 264 bytes in E4M3 (256 of codes, 8 of
// scales) and 136 in E2M1, read once for the rows of a tile; a unit costs a wavefront as many vector operations to widen 32
// keys and values as two products of 16 rows take matrix cycles.  So wavefronts have few rows and keys of their own: no key is
// widened twice, and nothing waits for a barrier while memory answers.  8 KV heads of 4 query heads, us (GB/s of codes and
// scales): a token of each of 16 sequences of up to 32768 in 8 bits 106, in 4 bits 74; 16 tokens of each 150, 122; one of
// 131072 in 8 bits 60 (4620), in 4 bits 41; a token of each of 16 of 4122 in 8 bits 31.6 (4420), where tiles of 128 rows that
// share keys through LDS took 74.  Of a short call 2 us find the places, 5 bring the first keys, 5 join the parts.
// Two units requested ahead, with 12 wavefronts in the place of 16, were 0.5 to 0.8 us faster where a workgroup has one round, and
// 2 to 5 % slower where it has many.
#include "chunk_attend_core.h"
#include "few_division.h"

namespace rkv {

namespace {

// Wavefronts of a SIMD: as many as the registers allow (128 of 512 each, 168, 256), all of one workgroup, so that a compute
// unit's keys are one stretch and its results are joined in LDS.
constexpr int few_per_simd(int tiles) { return tiles == 1 ? 4 : tiles == 2 ? 3 : 2; }
constexpr int few_waves(int tiles) { return 4 * few_per_simd(tiles); }
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

// How the tiles of a KV head are divided, and the piece a workgroup takes.
struct FewRow {
  int units, pieces, from, to;
  int size;  // of parts that no two tiles share, from .. to then being counted in parts; or 0
};
// The part of a tile that a piece holds, units u0 .. u1 - 1 of it.
struct FewPart {
  int b, row, n, len;       // the sequence, see ChunkSeq
  int tile, u0, u1, end;    // end: of the part in the row
  int part, parts, first;   // first: the piece that holds the tile's beginning
};

template <View VIEW>
__device__ __forceinline__ int few_tiles(const ChunkAttendArgs& a, const ChunkSeq& s) {
  return VIEW == kWhole ? 1 : chunk_ceil(s.n, a.tile_tokens);
}
__device__ __forceinline__ int few_units(const ChunkSeq& s) { return max(1, chunk_ceil(s.len, 32)); }  // (a tile without keys has one of none)

// Lists are all of one length, so the host knows how they are divided: units of one, parts of one (0: pieces of the row).
struct FewLists {
  int units, pieces, parts;
  Divider by_parts;
};
FewLists few_lists(int batch, int tokens, int slots) {
  FewLists l = {max(1, chunk_ceil(tokens, 32)), 0, 0, divider(1)};
  const int units = batch * l.units;
  for (int i = 0; i < few_tries(units, slots) && l.parts == 0; ++i) {
    const int parts = few_parts(l.units, few_size(units, slots, i));
    if ((int64_t)batch * parts <= slots) l.parts = parts;
  }
  l.pieces = l.parts ? batch * l.parts : few_pieces(units, batch, slots);
  l.by_parts = divider(l.parts ? l.parts : 1);
  return l;
}
__device__ __forceinline__ FewRow list_row(FewLists l, int batch, int at) {
  if (at >= l.pieces) return {0, 0, 0, 0, 0};
  const int units = batch * l.units;
  if (l.parts) return {units, l.pieces, at, at + 1, 0};
  return {units, l.pieces, few_begin(units, at, l.pieces), few_begin(units, at + 1, l.pieces), 0};
}
// Where place `from` of the row lies in its tile: `place` of its `parts` parts, or (0) of its units.
__device__ __forceinline__ void place_in(FewPart& p, FewRow r, int at, int from, int place, int units, int parts) {
  int u0 = place, u1, end, first = at - place, n = parts;
  if (parts == 1) {
    u1 = units, end = from + 1;
  } else if (parts) {
    u0 = few_begin(units, place, parts), u1 = few_begin(units, place + 1, parts), end = from + 1;
  } else {
    const int begin = from - place;
    end = min(r.to, begin + units), u1 = end - begin;
    first = few_piece_of(r.units, begin, r.pieces);
    n = few_piece_of(r.units, begin + units - 1, r.pieces) - first + 1;
  }
  p.u0 = u0, p.u1 = u1, p.end = end;
  p.part = at - first, p.parts = n, p.first = first;
}
__device__ __forceinline__ FewPart list_part(FewLists l, FewRow r, int tokens, int at, int from) {
  FewPart p;
  const int parts = l.parts, units = l.units;
  p.b = p.row = parts ? (int)divide((uint32_t)from, l.by_parts) : from / units;
  p.n = 1, p.len = tokens, p.tile = 0;
  place_in(p, r, at, from, from - p.b * (parts ? parts : units), units, parts);
  return p;
}

// Both by one wavefront, a sequence a lane; `own`: of the first 64, looked up once.
template <View VIEW>
__device__ __forceinline__ FewRow few_row(const CacheView& c, const ChunkAttendArgs& a, const ChunkSeq& own, int at) {
  const auto each = [&](const auto& count, int64_t* rows = nullptr) {  // the sum over all tiles of what count(units) says
    const int lane = threadIdx.x % kWave;
    uint32_t sum = 0;
    for (int b0 = 0; b0 < c.batch; b0 += kWave) {
      uint32_t x = 0, n = 0;
      if (b0 + lane < c.batch) {
        const ChunkSeq s = b0 == 0 ? own : chunk_seq<VIEW>(c, a, b0 + lane);
        n = (uint32_t)s.n;
        x = (uint32_t)few_tiles<VIEW>(a, s) * (uint32_t)count(few_units(s));
      }
      sum += (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(x), kWave - 1);
      if (rows) *rows += __builtin_amdgcn_readlane((int)wave_incl_scan(n), kWave - 1);
    }
    return (int)sum;
  };
  int64_t rows = 0;
  const int units = VIEW == kWhole ? each([](int u) { return u; }) : each([](int u) { return u; }, &rows);
  if (rows > a.ch.n_tokens) return {0, 0, 0, 0, 0};  // (more than was planned for, see few_bound)
  const int tries = few_tries(units, a.slots);
#pragma unroll 1
  for (int i = 0; i < tries; ++i) {
    const int size = few_size(units, a.slots, i), parts = each([&](int u) { return few_parts(u, size); });
    if (parts <= a.slots) return {units, parts, at, min(at + 1, parts), size};
  }
  const int pieces = few_pieces(units, each([](int) { return 1; }), a.slots);
  if (at >= pieces) return {units, pieces, 0, 0, 0};
  return {units, pieces, few_begin(units, at, pieces), few_begin(units, at + 1, pieces), 0};
}
template <View VIEW>
__device__ __forceinline__ FewPart few_part(const CacheView& c, const ChunkAttendArgs& a, const ChunkSeq& own, const FewRow& r, int at, int from) {
  FewPart p;
  ChunkSeq s;
  int idx;
  const auto share = [&](int u) { return r.size ? few_parts(u, r.size) : u; };  // of a tile in the row
  if (!locate_tile(c.batch, from, [&](int i) {
        const ChunkSeq s = i < kWave ? own : chunk_seq<VIEW>(c, a, i);
        return few_tiles<VIEW>(a, s) * share(few_units(s));
      }, p.b, idx))
    return FewPart{};  // (no rows; lengths that something else changes meanwhile)
  if (p.b < kWave) s = {__builtin_amdgcn_readlane(own.row, p.b), __builtin_amdgcn_readlane(own.n, p.b), __builtin_amdgcn_readlane(own.len, p.b)};
  else s = chunk_seq<VIEW>(c, a, p.b);
  const int u = few_units(s);
  p.row = s.row, p.n = s.n, p.len = s.len;
  const int of = share(u);
  p.tile = idx / of;
  place_in(p, r, at, from, idx - p.tile * of, u, r.size ? of : 0);
  return p;
}

}  // namespace

template <Source SRC, View VIEW, int NB>
__global__ __launch_bounds__(few_waves(NB) * kWave) __attribute__((amdgpu_waves_per_eu(few_per_simd(NB))))
void few_attend_kernel(CacheView c, ChunkAttendArgs a, uint32_t* counters, Divider by_page, FewLists all_lists) {
  constexpr int kRows = 16 * NB, kWaves = few_waves(NB);
  constexpr int kRowBytes = SRC == kE4M3 ? kHeadDim : kHeadDim / 2;
  constexpr int kKeyLoads = SRC == kE4M3 ? 2 : 1;  // of 16 bytes, a lane's 32 codes of a key
  typedef typename Codes16<SRC>::Raw Raw;
  extern __shared__ __align__(256) unsigned char s_tiles[];  // [wavefront] a unit's values; later a row tile's outputs
  __shared__ float s_stats[kWaves][kRows][3];  // later [half a wavefront] of those that join parts
  __shared__ u32x4 s_q[NB * 4 * kWave];
  __shared__ int s_last;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g = blockIdx.x % c.n_kv_heads, at = blockIdx.x / c.n_kv_heads;
  __shared__ FewRow s_row;
  __shared__ FewPart s_part;
  const int G = c.group, ps = c.page_size;
  __shared__ ChunkSeq s_own[kWave];
  const auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  // (lists are all of one length, and take no looking up)
  constexpr bool lists = VIEW == kListed;
  constexpr bool chunk = VIEW == kCausal || VIEW == kMasked;  // whose rows may see less than all keys of a tile
  FewRow whole = {0, 0, 0, 0, 0};
  if (lists) {
    const FewRow r = list_row(all_lists, c.batch, at);
    whole = {same(r.units), same(r.pieces), same(r.from), same(r.to), same(r.size)};
  } else if (wave == 0) {
    const int lane = threadIdx.x;
    const ChunkSeq own = chunk_seq_of_lane<VIEW>(c, a);
    s_own[lane] = own;
    const FewRow r = few_row<VIEW>(c, a, own, at);
    if (lane == 0) s_row = r;
    if (r.from < r.to) {
      const FewPart p = few_part<VIEW>(c, a, own, r, at, r.from);
      if (lane == 0) s_part = p;
    }
  }
  if (!lists) {
    __syncthreads();
    whole = {0, 0, same(s_row.from), same(s_row.to), 0};
  }
  const int to = whole.to;
#pragma unroll 1
  for (int from = whole.from; from < to;) {
    // (a lane's places are derived anew at each use: held over the loops they would take the registers that are left)
    const int tid = (int)use_late(threadIdx.x), lane = tid % kWave, i16 = lane % 16, kg = lane / 16;
    if (lists) asm volatile("" : "+s"(whole.units));  // (nor the reciprocals that divide by it)
    const FewPart found_part = lists ? list_part(all_lists, whole, a.row_len * ps, at, from) : s_part;
    const FewPart pl = {same(found_part.b), same(found_part.row), same(found_part.n), same(found_part.len), same(found_part.tile),
                        same(found_part.u0), same(found_part.u1), same(found_part.end), same(found_part.part),
                        same(found_part.parts), same(found_part.first)};
    if (!lists && pl.n == 0) return;
    const ChunkSeq s = {pl.row, pl.n, pl.len};
    from = pl.end;
    const int t0 = pl.tile * a.tile_tokens, nt = min(a.tile_tokens, s.n - t0);
    const int rows = nt * G;
    const int old = s.len - s.n, pos0 = old + t0;
    // its units that any row sees
    const int units = chunk_ceil(max(0, VIEW == kMasked ? s.len : min(s.len, pos0 + nt)), kUnit);
    const int u0 = pl.u0, u1 = min(pl.u1, units);

    const auto packed_row = [&](int r) {  // (token, head) of the packed tensors
      const int t = r / G;
      return (int64_t)(s.row + t0 + t) * c.n_q_heads + (int64_t)g * G + (r - t * G);
    };
    // The queries as every wavefront's lanes read them (from LDS, unit after unit: registers are what there is little of).
    // Requested here, put there once the first unit is under way as well.
    constexpr int kQueries = NB * 4 * kWave, kEach = (kQueries + kWaves * kWave - 1) / (kWaves * kWave);
    u32x4 query[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int x = min(tid + i * kWaves * kWave, kQueries - 1), ln = x % kWave, j = x / kWave % 4, r = x / (4 * kWave) * 16 + ln % 16;
      const int channel = SRC == kE4M3 ? j / 2 * 64 + ln / 16 * 16 + j % 2 * 8 : ln / 16 * 32 + 8 * j;
      query[i] = *reinterpret_cast<const u32x4*>(a.q + packed_row(min(r, rows - 1)) * kHeadDim + channel);
      if (r >= rows) query[i] = (u32x4){0u, 0u, 0u, 0u};
    }
    const auto put_queries = [&]() {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (tid + i * kWaves * kWave < kQueries) s_q[tid + i * kWaves * kWave] = query[i];
    };
    if (kEach > 1) put_queries();  // (or at once, where that would take too many registers)
    const int sees_first = VIEW == kMasked ? old - 1 : pos0;  // the last key that all rows see

    // Where the tokens of a unit lie, lane i of the first 32 token i, looked up a unit ahead (and a list's pages two).
    // (Its slot in the page is derived again when it is requested: a register less over the loop.)
    const int list_len = VIEW == kListed ? min(max(c.seq_lens[pl.b], 0), c.pages_cap * ps) : 0;
    const auto fresh = [&]() { return use_late((uint32_t)lane); };
    const auto token = [&](int u) { return (uint32_t)(u * kUnit) + fresh() % kUnit; };
    const auto list_entry = [&](int u) {
      const uint32_t t = token(u), p = divide(t, by_page);
      const int32_t* row = a.pages + ((int64_t)pl.b * c.n_kv_heads + g) * a.row_len;
      return u < u1 && (int)t < s.len ? row[p] : -1;
    };
    const auto find = [&](int u, int entry) {
      const uint32_t t = token(u), p = divide(t, by_page);
      if (VIEW == kListed) {
        const bool there = entry >= 0 && entry < c.pages_cap && entry * ps + (int)(t - p * ps) < list_len;
        return there ? phys_page_request(c, pl.b, entry) : -1;
      }
      return u < u1 && (int)t < s.len ? phys_page_request(c, pl.b, (int)p) : -1;
    };
    const auto in_range = [&](int raw) { return raw >= 0 && (int64_t)raw < c.n_phys_pages; };
    const auto place_of = [&](int u, int raw) {  // counted in tokens over the pool; that of an absent one is the first
      const uint32_t t = token(u), slot = t - divide(t, by_page) * (uint32_t)ps;
      return in_range(raw) ? (uint32_t)(raw * c.stride_page + g * c.stride_head) + slot : 0u;
    };

    u32x4 k_raw[2][kKeyLoads];
    uint32_t k_scale[2], v_scale[4];
    Raw v_raw[4];
    // Returns a bit per token that exists.  Values past the caches, keys through them: a key row's codes come in two requests or
    // lie beside the next row's, and the second finds its line there.  (16 tokens over 4122 in 8 bits and 64 listed pages of 16
    // sequences, us: both past 36.0 and 18.0, both through 37.2 and 15.3, so 34.2 and 16.0.)
    const auto request = [&](int u, int raw) {
      const uint32_t tok = place_of(u, raw), valid = (uint32_t)__ballot(in_range(raw));
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
      const uint32_t r = nb * 16 + fresh() % 16;
      if ((int)r >= rows) return 0u;
      const uint32_t t = r / (uint32_t)G;
      if (VIEW != kMasked) {
        const int n = pos0 + (int)t - key0 + 1;
        return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
      }
      const int j = key0 - old;
      if (j <= -32) return ~0u;
      const uint32_t* tile = a.mask + (int64_t)(s.row + t0) * a.mask_words;
      const int w = j >> 5, place = (int)t * a.mask_words + w;
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
    int entry = -1, found = -1;
    uint32_t valid = 0;
    if (u < u1) {
      if (VIEW == kListed) {
        const int e0 = list_entry(u), e1 = list_entry(u + kWaves);
        entry = list_entry(u + 2 * kWaves);
        const int f = find(u, e0);
        found = find(u + kWaves, e1);
        valid = request(u, f);
      } else {
        const int f = find(u, entry);
        found = find(u + kWaves, entry);
        valid = request(u, f);
      }
    }
    if (kEach == 1) put_queries();
    __syncthreads();
    if (!lists && wave == 0 && from < to) {  // (all have read where this part is)
      const FewPart p = few_part<VIEW>(c, a, s_own[fresh()], s_row, at, from);
      if (fresh() == 0) s_part = p;
    }
    for (; u < u1; u += kWaves) {
      const int key0 = u * kUnit;
      const uint32_t there = valid;
      // values to LDS: chunk x of row r at x ^ 4 (r % 4)
      const bool partly = there != ~0u || key0 + kUnit - 1 > sees_first, apart = chunk && partly;
      bool odd = false;
      {
        const uint32_t ln = fresh();
        // (rows 8 further turn alike)
        const uint32_t to = (uint32_t)(wave * kUnitBytes) + ln / 8 * 256 + (((2 * (ln % 8)) ^ (4 * (ln / 8 % 4))) * 16);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          u32x4 lo, hi;
          widen16(v_raw[p], __uint_as_float(v_scale[p] << 23), lo, hi);
          *reinterpret_cast<u32x4*>(s_tiles + (to + p * 2048)) = lo;
          *reinterpret_cast<u32x4*>(s_tiles + ((to ^ 16u) + p * 2048)) = hi;
        }
        if (partly) {
#pragma unroll 1
          for (uint32_t x = 0; x < 8; ++x) {  // (a lane's own pieces again)
            u32x4* at = reinterpret_cast<u32x4*>(s_tiles + ((to ^ (x & 1u) * 16u) + x / 2 * 2048));
            u32x4 v = *at;
            const uint32_t live = there >> (x / 2 * 8 + ln / 8) & 1u ? ~0u : 0u;  // (0 x NaN is not 0)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t none = apart ? no_numbers(v[e]) & live : 0u;
              v[e] &= live & ~none;
              odd |= none != 0u;
            }
            *at = v;
          }
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
      const auto request_next = [&]() {
        if (u + kWaves >= u1) return;
        valid = request(u + kWaves, found);
        found = find(u + 2 * kWaves, entry);
        if (VIEW == kListed) entry = list_entry(u + 3 * kWaves);
      };
      if (NB < 4) request_next();
      u32x4 pf[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (partly) {  // (rows that are not there see what they like)
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
      if (NB >= 4) request_next();  // (the logits' registers are free now, which their places in memory take)
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
    if (chunk && odd_from >= 0) {
#pragma unroll 1
      for (u = odd_from; u < u1; u += kWaves) {
        const int key0 = u * kUnit;
        const uint32_t ln = fresh();
        const int raw = find(u, entry);
        const uint32_t tok = place_of(u, raw), there = (uint32_t)__ballot(in_range(raw));
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
    const auto part_at = [&](int part) {  // a piece has places for the tile it ends with, if that goes on, and the one it goes on with
      return (uint32_t)(((pl.first + part) * c.n_kv_heads + g) * 2 + (part == 0)) * kRows;
    };
    const uint32_t part_row = part_at(pl.part);
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
      for (int idx = (int)use_late(threadIdx.x); idx < min(rows - nb * 16, 16) * 32; idx += kWaves * kWave) {
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
    if (pl.parts == 1) {
      __syncthreads();  // (the next part's results come to the same places)
      continue;
    }

    // Whoever of the tile's workgroups is done last joins their results.  (See the hand-off of data between workgroups.)
    drain_stores();
    __syncthreads();
    uint32_t* counter = counters + pl.first * c.n_kv_heads + g;
    if ((int)use_late(threadIdx.x) == 0)
      s_last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)pl.parts - 1;
    __syncthreads();
    if (!s_last) continue;
    if ((int)use_late(threadIdx.x) == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // 32 lanes a row, as many threads beside each other on its parts as there are to spare
    constexpr int kSlots = kWaves * 2;
    const int share = max(1, kSlots / rows), slot = (int)use_late(threadIdx.x) / 32, q = (int)use_late(threadIdx.x) % 32;
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
            const uint32_t pr = part_at(ok ? p0 + x * share : p0) + r;
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
    __syncthreads();  // (as above)
  }
}

int64_t few_units_bound(const CacheView& c, int n_tokens, int tiles) {
  return few_bound(n_tokens, c.batch, 16 * tiles / c.group, (int64_t)c.pages_cap * c.page_size);
}

void plan_few(const CacheView& c, int n_tokens, int tiles, ChunkPlan& p) {
  p.far = p.stream = false;
  p.tile_rows = 16 * tiles;
  p.tile_tokens = p.tile_rows / c.group;
  int64_t most_tiles = (int64_t)n_tokens / p.tile_tokens + c.batch;
  if (most_tiles > n_tokens) most_tiles = n_tokens;
  p.slots = few_most((int)few_units_bound(c, n_tokens, tiles), (int)most_tiles, c.n_kv_heads < kFewMost ? kFewMost / c.n_kv_heads : 1);
  p.most = 2 * p.slots * c.n_kv_heads;
  p.cuts = p.slots > 1;
  p.workgroups = (int64_t)p.slots * c.n_kv_heads;
}

namespace {
template <View VIEW>
hipError_t launch_few(const QCacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, uint32_t* counters, hipStream_t st) {
  const int tiles = plan.tile_rows / 16;
  const FewLists lists = VIEW == kListed ? few_lists(c.tokens.batch, a.row_len * c.tokens.page_size, a.slots) : FewLists{0, a.slots, 0, {0, 0}};
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(lists.pieces * c.tokens.n_kv_heads)), dim3(few_waves(tiles) * kWave), few_waves(tiles) * kUnitBytes, st, c.tokens, a,
                       counters, divider(c.tokens.page_size), lists);
    return hipGetLastError();
  };
  const bool e4m3 = c.format == ROCKETKV_Q_E4M3;
  if constexpr (VIEW == kCausal || VIEW == kMasked) {
    if (tiles == 4) return e4m3 ? launch(few_attend_kernel<kE4M3, VIEW, 4>) : launch(few_attend_kernel<kE2M1, VIEW, 4>);
    if (tiles == 2) return e4m3 ? launch(few_attend_kernel<kE4M3, VIEW, 2>) : launch(few_attend_kernel<kE2M1, VIEW, 2>);
  }
  return e4m3 ? launch(few_attend_kernel<kE4M3, VIEW, 1>) : launch(few_attend_kernel<kE2M1, VIEW, 1>);
}

}  // namespace

hipError_t launch_few_attend(const QCacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, bool singles, uint32_t* counters,
                             hipStream_t st) {
  if (singles) return a.pages ? launch_few<kListed>(c, a, plan, counters, st) : launch_few<kWhole>(c, a, plan, counters, st);
  return a.mask ? launch_few<kMasked>(c, a, plan, counters, st) : launch_few<kCausal>(c, a, plan, counters, st);
}

}  // namespace rkv
