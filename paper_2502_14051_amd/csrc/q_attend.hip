// Attention over quantised caches: of a chunk of new tokens, and of single tokens over a list of pages.
//
// Keys and values are widened to bf16 on their way into LDS, which is exact (a code of at most four significant bits times
// a power of two), so what follows is the attention over bf16 caches that hold the same values.
#include "chunk_attend_core.h"

namespace rkv {

// Rows of a sequence on average up to which its keys are walked by wavefronts of their own.
constexpr int kFewRows = 64;

ChunkPlan plan_q_attend(const QCacheView& c, int n_tokens) {
  ChunkPlan p;
  const int64_t rows = (int64_t)n_tokens * c.tokens.group / c.tokens.batch;
  p.far = p.stream = false;
  p.tile_rows = rows <= 128 ? 128 : 256;
  plan_chunk_tiles(c.tokens, n_tokens, p);
  const int tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  if (rows <= kFewRows && few_units_bound(c.tokens, n_tokens, tiles) < 1ll << 31) plan_few(c.tokens, n_tokens, tiles, p);
  return p;
}

ChunkPlan plan_q_list(const QCacheView& c, int row_len) {
  ChunkPlan p;
  p.tile_rows = 256;
  plan_chunk_tiles(c.tokens, c.tokens.batch, p);  // (for the size of its workspace)
  CacheView v = c.tokens;
  if (row_len > 0) v.pages_cap = row_len;
  plan_few(v, v.batch, 1, p);
  return p;
}

namespace {
template <Source SRC, View VIEW>
void launch_q(const CacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, hipStream_t st) {
  const auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.workgroups), dim3(waves * kWave), 4 * kKeyBytes, st, c, a);
  };
  if (plan.tile_rows == 256) launch(chunk_attend_kernel<SRC, false, 8, false, VIEW>, 8);
  else launch(chunk_attend_kernel<SRC, false, 4, false, VIEW>, 4);
}
ChunkAttendArgs q_attend_args(const QCacheView& c, const ChunkView& ch, const bf16_t* q, bf16_t* out, float* out_lse, void* ws,
                              const ChunkPlan& plan) {
  ChunkAttendArgs a = chunk_attend_args(ch, q, out, out_lse, ws, plan);
  a.k_scales = reinterpret_cast<const uint32_t*>(c.k_scales);
  a.v_scales = reinterpret_cast<const uint32_t*>(c.v_scales);
  return a;
}
}  // namespace

hipError_t launch_q_attend(const QCacheView& c, const ChunkView& ch, const MaskView& mask, const bf16_t* q, bf16_t* out,
                           float* out_lse, void* ws, const ChunkPlan& plan, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  ChunkAttendArgs a = q_attend_args(c, ch, q, out, out_lse, ws, plan);
  a.mask = mask.bits;
  a.mask_words = mask.words;
  if (plan.tile_rows <= kFewRows) return launch_few_attend(c, a, plan, false, static_cast<uint32_t*>(ws), st);
  if (c.format == ROCKETKV_Q_E4M3) mask.bits ? launch_q<kE4M3, kMasked>(c.tokens, a, plan, st) : launch_q<kE4M3, kCausal>(c.tokens, a, plan, st);
  else mask.bits ? launch_q<kE2M1, kMasked>(c.tokens, a, plan, st) : launch_q<kE2M1, kCausal>(c.tokens, a, plan, st);
  return launch_chunk_merge(c.tokens, a, plan, st);
}

hipError_t launch_q_list(const QCacheView& c, const int32_t* pages, int row_len, const bf16_t* q, bf16_t* out,
                         float* out_lse, void* ws, const ChunkPlan& plan, hipStream_t st) {
  ChunkAttendArgs a = q_attend_args(c, {c.tokens.batch, nullptr}, q, out, out_lse, ws, plan);
  a.pages = pages;
  a.row_len = row_len;
  return launch_few_attend(c, a, plan, true, static_cast<uint32_t*>(ws), st);
}

}  // namespace rkv
