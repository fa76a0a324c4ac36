// Attention over quantised caches: of a chunk of new tokens, and of single tokens over a list of pages.
//
// Keys and values are widened to bf16 on their way into LDS, which is exact (a code of at most four significant bits times
// a power of two), so what follows is the attention over bf16 caches that hold the same values.
#include "chunk_attend_core.h"

namespace rkv {

ChunkPlan plan_q_attend(const QCacheView& c, int n_tokens) {
  ChunkPlan p;
  p.far = false;
  p.stream = false;
  p.tile_rows = 256;
  plan_chunk_tiles(c.tokens, n_tokens, p);
  return p;
}

namespace {
template <Source SRC, View VIEW>
void launch_q(const CacheView& c, const ChunkAttendArgs& a, const ChunkPlan& plan, hipStream_t st) {
  hipLaunchKernelGGL((chunk_attend_kernel<SRC, false, 8, false, VIEW>), dim3((unsigned)plan.workgroups), dim3(8 * kWave), 4 * kKeyBytes, st, c, a);
}
template <View VIEW>
hipError_t launch_format(const QCacheView& c, ChunkAttendArgs a, const ChunkPlan& plan, hipStream_t st) {
  a.k_scales = reinterpret_cast<const uint32_t*>(c.k_scales);
  a.v_scales = reinterpret_cast<const uint32_t*>(c.v_scales);
  if (c.format == ROCKETKV_Q_E4M3) launch_q<kE4M3, VIEW>(c.tokens, a, plan, st);
  else launch_q<kE2M1, VIEW>(c.tokens, a, plan, st);
  return launch_chunk_merge(c.tokens, a, plan, st);
}
}  // namespace

hipError_t launch_q_attend(const QCacheView& c, const ChunkView& ch, const MaskView& mask, const bf16_t* q, bf16_t* out,
                           float* out_lse, void* ws, const ChunkPlan& plan, hipStream_t st) {
  if (ch.n_tokens == 0) return hipSuccess;
  ChunkAttendArgs a = chunk_attend_args(ch, q, out, out_lse, ws, plan);
  a.mask = mask.bits;
  a.mask_words = mask.words;
  return mask.bits ? launch_format<kMasked>(c, a, plan, st) : launch_format<kCausal>(c, a, plan, st);
}

ChunkPlan plan_q_list(const QCacheView& c, int row_len) {
  QCacheView v = c;
  v.tokens.pages_cap = row_len;
  return plan_q_attend(v, c.tokens.batch);
}

hipError_t launch_q_list(const QCacheView& c, const int32_t* pages, int row_len, const bf16_t* q, bf16_t* out,
                         float* out_lse, void* ws, const ChunkPlan& plan, hipStream_t st) {
  ChunkAttendArgs a = chunk_attend_args({c.tokens.batch, nullptr}, q, out, out_lse, ws, plan);
  a.pages = pages;
  a.row_len = row_len;
  return launch_format<kListed>(c, a, plan, st);
}

}  // namespace rkv
