// Attention of a chunk over bf16 caches: the kernel's forms for them, and how its parts are joined.
#include "chunk_attend_core.h"

namespace rkv {

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
  p.stream = chunk_past_caches(p.far, rows, held);
  plan_chunk_tiles(c, n_tokens, p);
  return p;
}

void plan_chunk_tiles(const CacheView& c, int n_tokens, ChunkPlan& p) {
  p.tile_tokens = p.tile_rows / c.group;
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
}

ChunkAttendArgs chunk_attend_args(const ChunkView& ch, const bf16_t* q, bf16_t* out, float* out_lse, void* ws,
                                  const ChunkPlan& plan) {
  ChunkAttendArgs a = {};
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
  return a;
}

hipError_t launch_chunk_merge(const CacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, hipStream_t st) {
  if (plan.cuts)
    hipLaunchKernelGGL(chunk_merge_kernel, dim3(plan.most, kMergeSlices), dim3(kMergeWaves * kWave), 0, st, c, a, plan.tile_rows);
  return hipGetLastError();
}

namespace {
template <View VIEW>
void launch_view(const CacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, hipStream_t st) {
  const auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.workgroups), dim3(waves * kWave), 4 * kKeyBytes, st, c, a);
  };
  if (plan.far) launch(chunk_attend_kernel<kByToken, true, 8, false, VIEW>, 8);
  else if (plan.tile_rows == 256 && c.v_token_major) launch(chunk_attend_kernel<kByToken, false, 8, false, VIEW>, 8);
  else if (plan.tile_rows == 256) launch(chunk_attend_kernel<kByChannel, false, 8, false, VIEW>, 8);
  else if (c.v_token_major && plan.stream) launch(chunk_attend_kernel<kByToken, false, 4, true, VIEW>, 4);
  else if (c.v_token_major) launch(chunk_attend_kernel<kByToken, false, 4, false, VIEW>, 4);
  else if (plan.stream) launch(chunk_attend_kernel<kByChannel, false, 4, true, VIEW>, 4);
  else launch(chunk_attend_kernel<kByChannel, false, 4, false, VIEW>, 4);
}
}  // namespace

hipError_t launch_chunk_attend(const CacheView& c, const ChunkView& ch, const MaskView& mask, const bf16_t* q, bf16_t* out,
                               float* out_lse, void* ws, const ChunkPlan& plan, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  ChunkAttendArgs a = chunk_attend_args(ch, q, out, out_lse, ws, plan);
  a.mask = mask.bits;
  a.mask_words = mask.words;
  if (mask.bits) launch_view<kMasked>(c, a, plan, st);
  else launch_view<kCausal>(c, a, plan, st);
  return launch_chunk_merge(c, a, plan, st);
}

}  // namespace rkv
