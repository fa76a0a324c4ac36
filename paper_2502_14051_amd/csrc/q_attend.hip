// Attention over quantised caches: of a chunk of new tokens, and of single tokens over a list of pages.
//
// Keys and values are widened to bf16 on their way into LDS, which is exact (a code of at most four significant bits times
// a power of two), so what follows is the attention over bf16 caches that hold the same values.  The matrix cores also take
// codes with their powers of two as they are, at twice to four times the rate; but they add such products with about 13 bits
// (sums of 128 products were up to 2e-4 of their magnitudes off, bf16 ones 1e-7), queries and weights would have to become
// codes too, and what most calls wait for is memory.
//
// Two forms.  Few rows: wavefronts with keys of their own (the attention of few rows, beside).  Many: tiles of 128 or 256 rows
// that share every key through LDS, as over bf16 caches, but with codes requested to registers two steps ahead and widened on
// their way to LDS, which costs vector operations beside the exponentials' (2048 tokens behind 32768, 4 heads to a KV head: 1092
// us from 4 bits, 1040 to 1118 from bf16).
#include "chunk_attend_core.h"

namespace rkv {

// Rows of a sequence on average up to which its keys are walked by wavefronts of their own.  us that way, in tiles of 128 and of
// 256 rows, 8 KV heads of 4 query heads: 9 tokens of each of 16 sequences of 4096 in 8 bits 46, 62, 76; 16 of each of up to 32768
// 150, 200, 200.  64 rows at most: the sums of twice as many do not fit a wavefront's registers.
constexpr int kFewRows = 64;
// Rows on average up to which tiles have 128 rows.  us in tiles of 128 and of 256: 32 tokens of each of 16 sequences of up to
// 32768 in 8 bits 188, 275; 100 behind 8000 43, 40; 387 behind 131072 1178, 951; 2048 behind 32768 in 4 bits 1226, 1092.
constexpr int kSmallTile = 128;
// Tokens a sequence has room for up to which they do too, as it is workgroups that such short rows of keys lack: prompts of up
// to 472 of one head 20.3, 24.2; 200 behind 1000 in 4 bits 24.2, 28.9; 64 of each of 16 behind 1000 46, 52; 2000 alone in 8 bits
// 76, 78; but 4000 alone in 4 bits 182, 167, 8000 in 8 bits 607, 565, 500 behind 4000 68, 65.
constexpr int kShortCache = 2048;

ChunkPlan plan_q_attend(const QCacheView& c, int n_tokens) {
  ChunkPlan p;
  const int64_t rows = (int64_t)n_tokens * c.tokens.group / c.tokens.batch;
  p.far = p.stream = false;
  p.tile_rows = rows <= kSmallTile || (int64_t)c.tokens.pages_cap * c.tokens.page_size <= kShortCache ? 128 : 256;
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
