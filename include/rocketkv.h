/*
 * rocketkv.h -- C ABI of the MI355X (gfx950) RocketKV hot path.
 *
 * RocketKV (arXiv 2502.14051) compresses the KV cache of a decoder LLM in two
 * stages: a one-time, GQA-aware SnapKV eviction of prompt tokens (Section 3.3)
 * and, at every decode step, hybrid sparse attention (HSA, Section 3.4 and
 * Algorithm 1): page-wise min/max key summaries, a top-k1 channel pick per GQA
 * group, approximate page scores, a top-k page pick and exact attention over
 * the picked pages only.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - All data pointers are DEVICE pointers unless marked "host".  The struct
 *    `rocketkv_cache_t` itself lives in host memory and is read during the
 *    call only.
 *  - bf16 tensors are passed as `void*` / `const void*` (2 bytes per element,
 *    upper half of an IEEE binary32).
 *  - `stream` is a `hipStream_t` passed as `void*` (NULL = the null stream).
 *    Work is enqueued on it and the call returns without synchronising.  No
 *    entry point allocates or frees device memory; scratch comes from the
 *    caller's `workspace` (size from rocketkv_workspace_bytes, 256-byte
 *    aligned).  A workspace must be passed once through
 *    rocketkv_workspace_init after it is allocated, and again whenever it is
 *    reused for a cache of a different shape; every call leaves it ready for
 *    the next.  Two calls that overlap in time must not share one.
 *  - Return value: ROCKETKV_OK (0) or a negative rocketkv_status_t.  Argument
 *    validation runs on the host before anything is launched; on error
 *    nothing has been enqueued and rocketkv_last_error() describes the
 *    reason (thread-local, valid until the next call on the same thread).
 *  - The caller owns every buffer.  The library keeps no state between calls.
 *
 * Cache layout (chosen for CDNA4 matrix-core operand order)
 * ---------------------------------------------------------
 * A cache is a pool of physical pages of `page_size` tokens.  For a physical
 * page `pp` and KV head `g` the tile starts at element
 *        pp * stride_page + g * stride_head
 * of the pool and holds `page_size * head_dim` contiguous bf16 values:
 *        K tile: [page_size][head_dim]   (token-major, channels contiguous)
 *        V tile: [head_dim][page_size]   (channel-major, tokens contiguous) when
 *                v_layout == ROCKETKV_V_CHANNEL_MAJOR, else [page_size][head_dim]
 * The channel-major V tile with page_size 16 is the layout the fused decode
 * kernel is built for (the token index is the contraction index of its second
 * matrix product).  The token-major V tile keeps every token's value row
 * contiguous, which is what page sizes other than 16 (Section 3.6 derives 2-4
 * for the usual budgets) and token-granular gathers need.
 * Sequence b's logical page p (tokens p*page_size ...) is physical page
 * `block_table[b*pages_cap + p]`, or `b*pages_cap + p` when block_table is
 * NULL.  `seq_lens[b]` is the number of valid tokens of sequence b (all KV
 * heads of a sequence hold the same number of tokens).  Entries of the block
 * table outside [0, n_phys_pages) are treated as absent pages.
 *
 * Page summaries (Section 3.4 Step 1) are two bf16 tensors
 *        kmax, kmin: [batch][n_kv_heads][head_dim][pages_cap]
 * i.e. channel-major with the page index contiguous, so that each channel
 * picked in Step 2 is one contiguous row.  Columns >= ceil(seq_len/page_size)
 * are never read.
 *
 * Limits of this build: head_dim == 128; n_q_heads a multiple of n_kv_heads
 * with group size <= 16; page_size 1..64, and 16 where V is channel-major and
 * attention or SnapKV is involved; pages_cap a multiple of 8 and at most
 * ROCKETKV_MAX_PAGES for selection.
 */
#ifndef ROCKETKV_H
#define ROCKETKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ROCKETKV_MAX_PAGES 32768

typedef enum {
  ROCKETKV_OK = 0,
  ROCKETKV_INVALID_ARG = -1,         /* NULL pointer, bad shape, bad budget ...      */
  ROCKETKV_UNSUPPORTED = -2,         /* valid request outside this build's limits    */
  ROCKETKV_WORKSPACE_TOO_SMALL = -3, /* workspace_bytes < rocketkv_workspace_bytes() */
  ROCKETKV_HIP_ERROR = -4            /* a HIP runtime call failed                    */
} rocketkv_status_t;

typedef enum {
  ROCKETKV_OP_HSA_DECODE = 0,   /* a = token_budget                       */
  ROCKETKV_OP_DENSE_DECODE = 1, /* no extra arguments                     */
  ROCKETKV_OP_SNAPKV = 2,       /* a = window, b = keep_budget            */
  ROCKETKV_OP_ATTEND = 3,       /* a = pages_row_len (0 = every page)     */
  ROCKETKV_OP_APPEND_CHUNK = 4, /* a = n_tokens                           */
  ROCKETKV_OP_CHUNK_ATTEND = 5, /* a = n_tokens                           */
  ROCKETKV_OP_WEIGHT_EVICT = 6  /* a = n_recent, b = keep_budget          */
} rocketkv_op_t;

typedef enum {
  ROCKETKV_V_CHANNEL_MAJOR = 0, /* V tile [head_dim][page_size] */
  ROCKETKV_V_TOKEN_MAJOR = 1    /* V tile [page_size][head_dim] */
} rocketkv_v_layout_t;

typedef struct rocketkv_cache {
  int32_t batch;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t page_size;
  int32_t pages_cap;          /* logical pages per sequence: row length of block_table / summaries */
  int64_t n_phys_pages;       /* pages in the pools */
  int64_t stride_page;        /* elements between physical pages (same for K and V pools) */
  int64_t stride_head;        /* elements between KV heads inside a page, >= page_size*head_dim */
  int32_t* seq_lens;          /* device [batch]; written by snapkv_compress (dst) and append_kv */
  const int32_t* block_table; /* device [batch][pages_cap] or NULL (identity) */
  void* k_pool;               /* device bf16 */
  void* v_pool;               /* device bf16 */
  int32_t v_layout;           /* rocketkv_v_layout_t */
} rocketkv_cache_t;

#define ROCKETKV_WS_HEADER_BYTES 65536 /* leading part of a workspace that workspace_init clears */

/* Scratch bytes needed by an operation on `cache` (host struct; device
 * pointers inside it are not dereferenced).  Returns 0 for an invalid
 * request (see rocketkv_last_error). */
size_t rocketkv_workspace_bytes(int32_t op, const rocketkv_cache_t* cache, int32_t a, int32_t b);

/*
 * Prepares a freshly allocated workspace: clears its first
 * min(workspace_bytes, ROCKETKV_WS_HEADER_BYTES) bytes (the arrival counters of the
 * split attention merge) on `stream`.  The attention entry points restore that
 * state themselves at the end of every call.
 */
int32_t rocketkv_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/*
 * HSA Step 1 (Section 3.4): element-wise max and min of the keys of each page,
 * over the valid tokens of the page only, for logical pages
 * [first_page, first_page + n_pages) of every (sequence, KV head); n_pages < 0
 * means "through the last page".  Pages at or beyond ceil(seq_len/page_size)
 * are skipped.  Exact: results are bf16 values present in K.
 * kmax, kmin: device bf16 [batch][n_kv_heads][head_dim][pages_cap], written.
 */
int32_t rocketkv_build_page_summaries(const rocketkv_cache_t* cache, void* kmax, void* kmin,
                                      int32_t first_page, int32_t n_pages, void* stream);

/*
 * HSA Step 2 (Algorithm 1, i1 / g / P / s1 / i2): per (sequence, KV head)
 *   a[c] = sum over the group's heads of |q[h][c]|,  s[c] = sum of q[h][c]  (fp32, head order)
 *   i1   = the channel_budget channels with the largest a (ties: lower channel)
 *   score[p] = sum over c in i1 of s[c] * (s[c] >= 0 ? kmax[c][p] : kmin[c][p])   (fp32)
 *   i2   = the kp pages with the largest score (ties: lower page), where
 *          kp = P if token_budget >= seq_len, else max(1, min(P, token_budget / page_size)),
 *          P = ceil(seq_len / page_size); the last min(n_recent_pages, kp) pages are always in.
 * q: bf16 [batch][n_q_heads][head_dim].
 * out_pages: int32 [batch][n_kv_heads][pages_row_len], ascending page ids, -1 padded;
 *            pages_row_len must be >= min(pages_cap, ceil(token_budget / page_size)).
 * out_channels: optional int32 [batch][n_kv_heads][channel_budget], ascending.
 * out_scores: optional fp32 [batch][n_kv_heads][pages_cap] (first P entries written); required
 *             when pages_cap exceeds 8192 (the selection then runs as a score launch and a top-k
 *             launch with the scores in between; the decode entry points keep them in the workspace).
 */
int32_t rocketkv_hsa_select(const rocketkv_cache_t* cache, const void* q, const void* kmax,
                            const void* kmin, int32_t channel_budget, int32_t token_budget,
                            int32_t n_recent_pages, int32_t* out_pages, int32_t pages_row_len,
                            int32_t* out_channels, float* out_scores, void* stream);

/*
 * HSA Step 3 (Algorithm 1, y = attn(q, K[i2], V[i2])): exact softmax attention
 * (scale 1/sqrt(head_dim)) of every query head over the valid tokens of the
 * listed pages of its KV head; bf16 operands, fp32 accumulation, bf16 result
 * rounded to nearest even.
 * pages: int32 [batch][n_kv_heads][pages_row_len] logical page ids; entries
 *        < 0 or >= ceil(seq_len/page_size) are ignored.  NULL = every page of
 *        the sequence (full-KV attention, the Full-KV row of Table 1).
 * out: bf16 [batch][n_q_heads][head_dim]; a sequence with no attended token
 *      gets zeros.  out_lse: optional fp32 [batch][n_q_heads], natural-log
 *      sum-exp of the scaled logits (-inf when nothing was attended).
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_ATTEND, cache, pages_row_len, 0).
 */
int32_t rocketkv_attend(const rocketkv_cache_t* cache, const void* q, const int32_t* pages,
                        int32_t pages_row_len, void* out, float* out_lse, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * One HSA decode step over a cache whose summaries are current: Step 2 then
 * Step 3 (Algorithm 1 end to end).  Arguments as in rocketkv_hsa_select and
 * rocketkv_attend; out_pages (row length min(pages_cap, ceil(token_budget /
 * page_size))), out_channels and out_lse are optional.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_HSA_DECODE, cache, token_budget, 0).
 */
int32_t rocketkv_hsa_decode(const rocketkv_cache_t* cache, const void* q, const void* kmax,
                            const void* kmin, int32_t channel_budget, int32_t token_budget,
                            int32_t n_recent_pages, void* out, float* out_lse,
                            int32_t* out_pages, int32_t* out_channels, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * rocketkv_hsa_decode for callers that cannot allocate device memory or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.  Same arguments, same
 * kernels and the same results as rocketkv_hsa_decode, minus the workspace: the scratch memory (arrival
 * counters, split partials, the page list and page scores of the multi-launch paths) is a buffer of
 * ROCKETKV_NOALLOC_SCRATCH_BYTES that is part of the library's device code, one copy per GPU, held
 * until the process ends.  The call allocates and frees nothing.  It clears the buffer's counter
 * header with a small fill kernel on `stream` first, so it costs one short launch more than
 * rocketkv_hsa_decode.  A shape whose scratch need (rocketkv_workspace_bytes(ROCKETKV_OP_HSA_DECODE,
 * ...)) exceeds the buffer is refused with ROCKETKV_UNSUPPORTED.  Every call on a GPU uses that GPU's
 * one buffer: calls that overlap in time on one GPU (two streams, two threads) race and must be
 * serialised by the caller; calls on different GPUs are independent.  The device current at the call
 * must be the one `stream` and the buffers belong to.
 */
#define ROCKETKV_NOALLOC_SCRATCH_BYTES (4u << 20)
int32_t rocketkv_hsa_decode_noalloc(const rocketkv_cache_t* cache, const void* q, const void* kmax,
                                    const void* kmin, int32_t channel_budget, int32_t token_budget,
                                    int32_t n_recent_pages, void* out, float* out_lse,
                                    int32_t* out_pages, int32_t* out_channels, void* stream);

/*
 * One decode step including the token generated at it (Section 3.4 Step 1, last
 * sentence, then Algorithm 1): the result, the caches, the summaries and
 * seq_lens end up exactly as after rocketkv_append_kv(k_new, v_new) followed by
 * rocketkv_hsa_decode, in one launch where the shapes allow.  kmax / kmin are
 * read and written.  k_new, v_new: bf16 [batch][n_kv_heads][head_dim].
 * workspace: as for rocketkv_hsa_decode (same size, same initialisation).
 */
int32_t rocketkv_hsa_decode_append(const rocketkv_cache_t* cache, const void* q, const void* k_new,
                                   const void* v_new, void* kmax, void* kmin, int32_t channel_budget,
                                   int32_t token_budget, int32_t n_recent_pages, void* out,
                                   float* out_lse, int32_t* out_pages, int32_t* out_channels,
                                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * Full-KV decode attention (Table 1, first row; the baseline every figure of
 * Section 4.3 is normalised to): rocketkv_attend with every page.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_DENSE_DECODE, cache, 0, 0).
 */
int32_t rocketkv_dense_decode(const rocketkv_cache_t* cache, const void* q, void* out,
                              float* out_lse, void* workspace, size_t workspace_bytes,
                              void* stream);

/*
 * Appending one generated token per sequence (Section 3.4 Step 1, last
 * sentence: the summaries follow every new key): writes k_new / v_new
 * (bf16 [batch][n_kv_heads][head_dim]) at position seq_lens[b], folds the key
 * into the tail page's kmax / kmin, then increments seq_lens[b].  A sequence
 * already holding pages_cap * page_size tokens is left unchanged.
 */
int32_t rocketkv_append_kv(const rocketkv_cache_t* cache, const void* k_new, const void* v_new,
                           void* kmax, void* kmin, void* stream);

/*
 * Stage 1 (Section 3.3; window and kernel sizes from Appendix A.3): GQA-aware
 * SnapKV.  Per (sequence, KV head) with prompt length S = src->seq_lens[b]:
 *   if S <= keep_budget every token is kept; otherwise
 *   A[h][w][j] = causal softmax over j <= S-window+w of q_obs[h][w] . K[j] / sqrt(head_dim)
 *   vote[j] = sum over heads of the group and window rows of A[h][w][j],  j < S-window
 *   pooled  = stride-1 max-pool of vote with odd kernel pool_kernel, clipped at the ends
 *   kept    = top-(keep_budget - window) of pooled (ties: lower position) plus the window
 * and K/V of the kept tokens are copied, in ascending position, into `dst`
 * (same head counts and head_dim; dst->pages_cap*page_size >= keep_budget),
 * dst->seq_lens[b] = min(S, keep_budget).
 * q_obs: bf16 [batch][n_q_heads][window][head_dim], queries of the last
 *        `window` prompt positions.
 * src needs page_size 16; dst may have any page size when its V is token-major.
 * kept_idx: optional int32 [batch][n_kv_heads][keep_budget], -1 padded.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_SNAPKV, src, window, keep_budget), which never shrinks as
 *            src->pages_cap grows: one sized for the longest cache serves every shorter one.
 */
int32_t rocketkv_snapkv_compress(const void* q_obs, const rocketkv_cache_t* src, int32_t window,
                                 int32_t pool_kernel, int32_t keep_budget,
                                 const rocketkv_cache_t* dst, int32_t* kept_idx, void* workspace,
                                 size_t workspace_bytes, void* stream);

/*
 * RocketKV-MT (Section 3.5): the multi-turn variant.  Stage 1 evicts nothing: the cache keeps every
 * token of the conversation, and Stage 2 runs over the subset Stage 1 filtered for the current turn
 * plus the tokens generated since, reached through an index.  At the next turn the filter runs
 * again over the whole cache, so a token passed over in one turn can come back in a later one.
 *
 * rocketkv_index_t describes that subset, the "logical sequence" of a (sequence, KV head):
 *   token_index[b][g][j] = position in the cache of logical token j, ascending in j;
 *   n_indexed[b]         = number of logical tokens (the same for every KV head of a sequence);
 *   page_size, pages_cap = page size and page capacity of Stage 2 over the logical order: page p
 *                          holds logical tokens p*page_size ..; summaries are
 *                          [batch][n_kv_heads][head_dim][pages_cap].
 * token_index rows have pages_cap * page_size entries.  The struct lives in host memory; its
 * pointers are device pointers, written by rocketkv_snapkv_filter and the *_append calls.
 * The cache itself must have token-major V (a token's row is what is gathered); its own page size
 * is free.  A logical sequence is exactly what rocketkv_snapkv_compress would have copied out, so
 * every mt call computes what its counterpart computes on that compacted cache.
 */
typedef struct rocketkv_index {
  int32_t* token_index;
  int32_t* n_indexed;
  int32_t page_size;
  int32_t pages_cap;
} rocketkv_index_t;

/*
 * Stage 1 as a filter (Section 3.5): the selection of rocketkv_snapkv_compress on `src` (all of its
 * rules, arguments and limits apply) written to index->token_index / index->n_indexed instead of a
 * compacted copy; src is left untouched.  Needs index->pages_cap * index->page_size >= keep_budget.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_SNAPKV, src, window, keep_budget).
 */
int32_t rocketkv_snapkv_filter(const void* q_obs, const rocketkv_cache_t* src, int32_t window,
                               int32_t pool_kernel, int32_t keep_budget, const rocketkv_index_t* index,
                               void* workspace, size_t workspace_bytes, void* stream);

/* rocketkv_build_page_summaries over the logical order of `index` (Section 3.4 Step 1 on the
 * filtered subset). */
int32_t rocketkv_mt_build_page_summaries(const rocketkv_cache_t* cache, const rocketkv_index_t* index,
                                         void* kmax, void* kmin, int32_t first_page, int32_t n_pages,
                                         void* stream);

/* Scratch bytes of rocketkv_mt_hsa_decode / rocketkv_mt_hsa_decode_append (0 on an invalid request). */
size_t rocketkv_mt_workspace_bytes(const rocketkv_cache_t* cache, const rocketkv_index_t* index,
                                   int32_t token_budget);

/*
 * rocketkv_hsa_decode over the logical sequence (Algorithm 1 restricted to the filtered subset):
 * selection on the logical pages, exact attention over the cache rows the picked logical tokens
 * point at.  out_pages holds logical page ids (row length min(index->pages_cap,
 * ceil(token_budget / index->page_size))).
 */
int32_t rocketkv_mt_hsa_decode(const rocketkv_cache_t* cache, const rocketkv_index_t* index,
                               const void* q, const void* kmax, const void* kmin,
                               int32_t channel_budget, int32_t token_budget, int32_t n_recent_pages,
                               void* out, float* out_lse, int32_t* out_pages, int32_t* out_channels,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * A generated token enters both the cache (position cache->seq_lens[b], as rocketkv_append_kv does)
 * and the logical sequence (entry index->n_indexed[b] of every KV head's index row, and the logical
 * tail page's kmax / kmin); both lengths grow by one.  A sequence whose cache or index is full is
 * left unchanged.
 */
int32_t rocketkv_mt_append_kv(const rocketkv_cache_t* cache, const rocketkv_index_t* index,
                              const void* k_new, const void* v_new, void* kmax, void* kmin,
                              void* stream);

/* rocketkv_mt_append_kv followed by rocketkv_mt_hsa_decode: one decode step of RocketKV-MT. */
int32_t rocketkv_mt_hsa_decode_append(const rocketkv_cache_t* cache, const rocketkv_index_t* index,
                                      const void* q, const void* k_new, const void* v_new, void* kmax,
                                      void* kmin, int32_t channel_budget, int32_t token_budget,
                                      int32_t n_recent_pages, void* out, float* out_lse,
                                      int32_t* out_pages, int32_t* out_channels, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * A chunk: the new tokens of all sequences of a cache, packed one behind the other.  Row r of a packed
 * tensor is one token; rows starts[b] .. starts[b+1]-1 belong to sequence b, in order.  A sequence may bring
 * no row, one, or a whole prompt.  starts must ascend from >= 0 to <= n_tokens (others read and write nothing out of range,
 * but results and counters in the workspace are not defined then); rows in front of starts[0] and behind starts[batch] are
 * neither read nor written.  The struct lives in host memory, starts on the device.
 */
#define ROCKETKV_MAX_CHUNK (1 << 24)
typedef struct rocketkv_chunk {
  int32_t n_tokens;      /* rows of the packed tensors, at most ROCKETKV_MAX_CHUNK */
  const int32_t* starts; /* device [batch + 1] */
} rocketkv_chunk_t;

/*
 * Rotary positions: of the leading rot_dim channels of a head, pair i is turned by the angle
 * position * inv_freq[i]:
 *   (x, y) -> scale * (x cos - y sin, y cos + x sin)
 * where pair i is channels (i, i + rot_dim / 2), or (2i, 2i + 1) with `interleaved`; the other channels pass through.
 * Angles are formed and reduced in 64 bits, the rotation is computed in fp32 and rounded to bf16 once.
 */
typedef struct rocketkv_rope {
  int32_t rot_dim;        /* even, 2 .. head_dim */
  int32_t interleaved;    /* 0 or 1 */
  const double* inv_freq; /* device [rot_dim / 2]: radians per position */
  float scale;            /* factor of the turned channels, 1 without scaling */
} rocketkv_rope_t;

/*
 * Frequencies for rotary positions, stretched for contexts longer than a model was trained on (host arithmetic in double
 * precision).  With f[i] = theta^(-2i / rot_dim):
 *   PLAIN   f[i]
 *   LINEAR  f[i] / factor                             positions interpolated
 *   BASE    theta replaced by theta * factor^(rot_dim / (rot_dim - 2)): the lowest frequency divided by factor, the
 *           highest unchanged (rot_dim > 2)
 *   BANDS   by turns t = original * f[i] / 2 pi over the original context: f[i] where t >= high, f[i] / factor where
 *           t <= low, and between them (1 - u) f[i] / factor + u f[i], u = (t - low) / (high - low)
 *   RAMP    the same mixture by the pair's index: u = 1 - clamp((i - a) / (b - a), 0, 1) where a, b are the indices at
 *           which a frequency makes `high` and `low` turns, rounded down and up, in [0, rot_dim - 1] (b at least
 *           a + 0.001); *scale = 0.1 ln(factor) + 1
 * *scale is 1 but for RAMP.  factor >= 1; BANDS and RAMP need 0 < low < high and original >= 1.
 */
typedef enum {
  ROCKETKV_ROPE_PLAIN = 0,
  ROCKETKV_ROPE_LINEAR = 1,
  ROCKETKV_ROPE_BASE = 2,
  ROCKETKV_ROPE_BANDS = 3,
  ROCKETKV_ROPE_RAMP = 4
} rocketkv_rope_kind_t;
int32_t rocketkv_rope_frequencies(int32_t kind, int32_t rot_dim, double theta, double factor, double low, double high,
                                  int64_t original, double* inv_freq /* host [rot_dim / 2] */, float* scale /* host */);

/*
 * Rotary positions of packed head rows: head h of token t is at x + t * x_stride + h * head_dim and goes to
 * y + t * y_stride + h * head_dim (bf16, head_dim 128; strides in elements, multiples of 8 and at least
 * n_heads * head_dim; x and y 16-byte aligned).  x == y with equal strides turns in place; other overlaps are not
 * allowed.  positions: device int32 [n_tokens], any value.
 */
int32_t rocketkv_rope(const rocketkv_rope_t* rope, const int32_t* positions, int32_t n_tokens, int32_t n_heads,
                      const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream);

/*
 * A chunk's tokens into the cache: token i of sequence b goes to position seq_lens[b] + i, its key turned by `rope`
 * (NULL: as it is), and seq_lens[b] grows by the sequence's rows.  The caches, summaries and lengths end up as after
 * rocketkv_append_kv of the (turned) tokens one by one, but that a sequence without room for all of its rows is left
 * unchanged.  Where q is given, the queries of all rows are turned into q_out as well.
 * q: bf16, token r at q + r * q_stride (n_q_heads heads); q_out: bf16 [n_tokens][n_q_heads][head_dim], may be q itself if
 *    q_stride is n_q_heads * head_dim; both NULL: no queries.
 * k_new, v_new: bf16, token r at + r * k_stride / v_stride (n_kv_heads heads).  Strides as in rocketkv_rope, so that all
 *    three may lie in the rows of one joint projection.
 * positions: device int32 [n_tokens] or NULL: a token's position in the cache (after an eviction the two differ).
 * kmax, kmin: both, or both NULL where no summaries are kept (RocketKV-MT builds them from the next filter).
 * Channel-major V needs page_size 16.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_APPEND_CHUNK, cache, n_tokens, 0).
 */
int32_t rocketkv_append_chunk(const rocketkv_cache_t* cache, const rocketkv_chunk_t* chunk, const rocketkv_rope_t* rope,
                              const int32_t* positions, const void* q, int64_t q_stride, void* q_out, const void* k_new,
                              int64_t k_stride, const void* v_new, int64_t v_stride, void* kmax, void* kmin,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * Causal attention of a chunk whose tokens are in the cache already: row i of the n rows of sequence b attends to the
 * tokens at positions 0 .. seq_lens[b] - n + i (scale 1/sqrt(head_dim)); bf16 operands, fp32 logits, softmax and sums,
 * weights rounded to bf16 for their product with the values, bf16 result.  Whole prompts (seq_lens[b] == n), pieces of prompts, turns and single tokens mix freely.
 * q, out: bf16 [n_tokens][n_q_heads][head_dim].  out_lse: optional fp32 [n_tokens][n_q_heads], natural-log sum-exp of the
 * scaled logits.  Absent pages are skipped; a row with nothing to attend to gets zeros and -inf, and one with a logit that
 * is NaN or +inf gets NaN in both.
 * Keys and values of a row's future, and whatever lies where no token is, may be anything.
 * out must not overlap q.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_CHUNK_ATTEND, cache, n_tokens, 0): 98 MiB for any n_tokens >= 1, so one
 * serves calls of any size.
 */
int32_t rocketkv_chunk_attend(const rocketkv_cache_t* cache, const rocketkv_chunk_t* chunk, const void* q, void* out,
                              float* out_lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The attention weight every cached token has received so far:
 *   weights_out[b][g][j] = (j < seq_lens[b] - n ? weights_in[b][g][j] : 0)
 *                        + sum over the group's heads h and the chunk's rows i that see j of
 *                          exp(q[i][h] . K[j] / sqrt(head_dim) - lse[i][h])
 * for j < seq_lens[b]; later entries are left as they were.  weights: fp32 [batch][n_kv_heads][pages_cap * page_size].
 * weights_in NULL counts as zeros and may be weights_out itself.  q and lse: as given to and left by
 * rocketkv_chunk_attend (or, with a chunk of one token per sequence, by rocketkv_dense_decode); a row whose lse is -inf
 * adds nothing whatever its query holds, nor does a token in an absent page receive any.  A row whose lse is NaN makes the
 * weights of the tokens that it sees NaN, and no others.
 */
int32_t rocketkv_accumulate_weights(const rocketkv_cache_t* cache, const rocketkv_chunk_t* chunk, const void* q,
                                    const float* lse, const float* weights_in, float* weights_out, void* stream);

/*
 * Eviction by accumulated weight.  Per (sequence, KV head) of S = src->seq_lens[b] tokens: all are kept if
 * S <= keep_budget; otherwise the last n_recent tokens and, of the others, the keep_budget - n_recent with the largest
 * weight (ties: lower position; NaN counts as larger than every number).  K, V and weights of the kept tokens go to
 * `dst`, in ascending position, and dst->seq_lens[b] = min(S, keep_budget).  src is left as it is.  A kept token whose page
 * is absent in src takes a place in dst like any other, with zeros for key and value (and its weight): from there on it is
 * a token, where attention over src skipped it.  A token of an absent page of dst goes nowhere.  A sequence longer than src
 * counts as empty.  A channel-major dst gets whole tiles, zeros behind the last token.
 * weights: fp32 [batch][n_kv_heads][src->pages_cap * src->page_size], 16-byte aligned.
 * dst: a cache with pools and lengths of its own, the same head counts, room for keep_budget tokens, any page size and
 *      V layout (channel-major: page_size 16, for src as well).
 * dst_weights: optional fp32 [batch][n_kv_heads][dst->pages_cap * dst->page_size], distinct from weights; the first
 *      min(S, keep_budget) entries of a row are written.
 * kept_idx: optional int32 [batch][n_kv_heads][keep_budget], -1 padded.
 * workspace: rocketkv_workspace_bytes(ROCKETKV_OP_WEIGHT_EVICT, src, n_recent, keep_budget).
 */
int32_t rocketkv_weight_evict(const rocketkv_cache_t* src, const float* weights, int32_t n_recent, int32_t keep_budget,
                              const rocketkv_cache_t* dst, float* dst_weights, int32_t* kept_idx, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * Adaptive compression decomposition (Section 3.6): for a sequence of seq_len
 * tokens and a total token budget t (memory traffic of one attention call in
 * key/value pairs, Step 2 and Step 3 together), c = seq_len / t (at least 1),
 *   r = min(0.2 + 0.06 log2 c, 0.8),  stage1 = c^r,  stage2 = c^(1-r),
 *   page_size = ceil(c^((1-r)/2)),  head_ratio = stage2 / page_size,
 * and, with the budget split evenly between Step 2 and Step 3 (Appendix A.3),
 *   keep_budget    = round(seq_len / stage1)          tokens Stage 1 keeps,
 *   channel_budget = round(head_dim / head_ratio)     in [1, head_dim],
 *   attend_tokens  = max(1, t / 2)                    the token_budget argument
 *                                                     of the decode entry points.
 * storage, storage_mt and traffic are the RocketKV and RocketKV-MT rows of Table 1 as printed:
 *   storage = 1/c^r + 2/c^((1+r)/2),  storage_mt = 1 + 2/c^((1+r)/2),  traffic = 1/c,
 * relative to the full KV cache; they bound what the buffers of this library need (the K_max /
 * K_min pair of a page size ps costs 1/ps of the kept K/V, half of Table 1's auxiliary term).
 * Host arithmetic only (double precision); `out` is a host struct.
 */
typedef struct rocketkv_split {
  double c, r, stage1, stage2, head_ratio;
  int32_t page_size, keep_budget, channel_budget, attend_tokens;
  double storage, storage_mt, traffic;
} rocketkv_split_t;
int32_t rocketkv_decompose(int64_t seq_len, int32_t token_budget, int32_t head_dim,
                           rocketkv_split_t* out);

/*
 * Measurement aid (no step of the method): read `bytes` (a multiple of 16) of device memory at
 * `src` (16-byte aligned) once, front to back, with plain streaming loads, and write one checksum
 * word per wavefront to `sink` (device, at least rocketkv_stream_read_sink_bytes() bytes).  Timed
 * over a buffer much larger than the 256 MB last-level cache it gives the read bandwidth this GPU
 * actually reaches, which the benchmark prints beside the published peak.  Asynchronous on `stream`.
 */
int32_t rocketkv_stream_read(const void* src, size_t bytes, void* sink, void* stream);
size_t rocketkv_stream_read_sink_bytes(void);

/*
 * Measurement aid (no step of the method): read the K and V tiles of the listed pages (the list
 * rocketkv_hsa_select writes: int32 [batch][n_kv_heads][pages_row_len], entries < 0 skipped) with the
 * work split and the load pattern of the attention kernels, and compute nothing: no logits, no
 * softmax, no merge.  Timed beside rocketkv_attend on the same list it gives the floor this GPU puts
 * under Step 3 (Algorithm 1, y = attn(q, K[i2], V[i2])) for that list: the gather of 4 KiB tiles
 * itself, plus one launch.  Channel-major V, 16-token pages.  `sink`: device, at least
 * rocketkv_stream_gather_sink_bytes(cache, pages_row_len) bytes, one checksum word per wavefront.
 * Asynchronous on `stream`.
 */
int32_t rocketkv_stream_gather(const rocketkv_cache_t* cache, const int32_t* pages, int32_t pages_row_len,
                               void* sink, void* stream);
size_t rocketkv_stream_gather_sink_bytes(const rocketkv_cache_t* cache, int32_t pages_row_len);

/* Thread-local description of the last error returned on this thread ("" if none). */
const char* rocketkv_last_error(void);

/* Library version, major*10000 + minor*100 + patch. */
int32_t rocketkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ROCKETKV_H */
