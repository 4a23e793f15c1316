/*
 * horizonserve_device.h -- operators of a decoding loop whose lengths, positions and page tables stay on the device.
 *
 * hs_stage_step takes its batch from the host: lengths and block tables are host arrays, and the host plans the work.  A loop
 * that is captured once in a CUDA graph, or whose next lengths the device itself decides, cannot do that.  The calls below
 * read every length, position and page id on the device, when they run:
 *     hs_op_step_tables      allocates the pages of a step and writes its per-token metadata
 *     hs_op_release_pages    gives the pages of finished requests back
 *     hs_op_rope_table       cos / sin of rotary positions, plain or stretched for long contexts
 *     hs_op_rope_cache       rotates q and k and scatters k and v into the paged cache
 *     hs_op_paged_attention  attention over the cache with capped scores, a distance bias, a window and a prefix
 *     hs_op_token_logprobs   log probabilities of given tokens, entropy and the top alternatives of logit rows
 * The pool, its pages and the free list's order are those of horizonserve.h (hs_kv_pool_bytes, hs_kv_alloc).  The paper has no
 * counterpart: it keeps its runtime's KV management and model execution (Sec. 5).
 *
 * Conventions are those of horizonserve.h: device pointers are borrowed, every call enqueues on the given stream and returns
 * without synchronising, no call allocates device memory, every kernel runs as at most sm_budget blocks of one per SM, and
 * results do not depend on sm_budget.  Besides
 *   - The description structs are read before the call returns; integers in them are element counts, strides count elements.
 *   - `status`: a device int, zero on entry, that receives an hs_status_t when a value that only the device knows is wrong
 *     (each call says which); the outputs are then as the call says.  It is left alone when nothing is wrong.  HS_ERR_TIMEOUT: a bounded wait inside
 *     a kernel ran out; the outputs are not defined, and the workspace is to be zeroed before its next use.
 *   - `workspace`: HS_DEVICE_WORKSPACE_BYTES of device memory, 256-byte aligned, zeroed once before its first use.  Every call
 *     leaves its control words at zero.  Two calls whose kernels can overlap on the GPU need two workspaces.
 *   - Errors that the host can see are returned and nothing is launched: INVALID_ARG (NULL, misaligned or inconsistent),
 *     UNSUPPORTED_SHAPE, INVALID_BUDGET, CUDA.
 */
#ifndef HORIZONSERVE_DEVICE_H_
#define HORIZONSERVE_DEVICE_H_

#include "horizonserve.h"

#ifdef __cplusplus
extern "C" {
#endif
#if defined(__GNUC__)
#pragma GCC visibility push(default)
#endif

#define HS_DEVICE_WORKSPACE_BYTES (32u << 20)
#define HS_DEVICE_MAX_SEQS 4096   /* requests of one call */
#define HS_MAX_ALTERNATIVES 32    /* top alternatives of a row */

/* Element types. */
#define HS_TYPE_F32 0
#define HS_TYPE_BF16 1
#define HS_TYPE_F16 2

/*
 * Page allocation and metadata of one step, from the requests' lengths.  Request s has ctx_len[s] tokens in the cache, which
 * own the first ceil(ctx_len[s] / 16) entries of its block table row, and q_len[s] >= 0 new ones.  In request order each request
 * pops the pages its new tokens need off the stack free_list (entry free_count - 1 first), exactly as hs_kv_alloc does on the
 * host.  Then, with tokens numbered request after request,
 *     tok_begin[s] = q_len[0] + .. + q_len[s - 1],   tok_begin[n_seqs] = tokens of the step,   kv_len[s] = ctx_len[s] + q_len[s],
 *     tok_seq[t] = s,   tok_pos[t] = ctx_len[s] + t - tok_begin[s],   tok_slot[t] = page * 16 + tok_pos[t] % 16,
 * and -1 in the per-token arrays from tok_begin[n_seqs] to max_tokens.  A step that cannot be done changes neither block_tables
 * nor the free list and describes a step without tokens (tok_begin 0, per-token arrays -1, kv_len = ctx_len), with the status
 *     OUT_OF_PAGES     the stack holds fewer pages than the step needs
 *     INVALID_ARG      a negative length, a request that outgrows its block table row, more than max_tokens tokens, or
 *                      free_count outside 0 .. num_pages
 * A page id outside 0 .. num_pages - 1, popped or owned, gives its tokens the slot -1 and the status BAD_BLOCK_TABLE; the step is done otherwise, a popped one is
 * in the block table, and hs_op_release_pages does not take it back.
 * kv_len may be ctx_len, and free_count_out may be free_count (a loop that advances in place); otherwise no arrays overlap.
 * n_seqs 1 .. HS_DEVICE_MAX_SEQS, n_seqs * max_pages_per_seq at most 2^27; a request has at most 2^31 - 64 tokens (here and in the calls below), however long its row.
 */
typedef struct {
  int32_t n_seqs, max_pages_per_seq, num_pages, max_tokens;
  const int32_t *ctx_len, *q_len; /* device [n_seqs] */
  const int32_t *free_list;       /* device [num_pages] */
  const int32_t *free_count;      /* device [1] */
  int32_t *block_tables;          /* device [n_seqs, max_pages_per_seq]: new entries are written, the others are kept */
  int32_t *kv_len;                /* device [n_seqs] */
  int32_t *tok_begin;             /* device [n_seqs + 1] */
  int32_t *tok_seq, *tok_pos, *tok_slot; /* device [max_tokens] */
  int32_t *free_count_out;        /* device [1] */
  void *workspace;
  int32_t *status;
} hs_step_tables_t;
hs_status_t hs_op_step_tables(const hs_step_tables_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Gives the pages of finished requests back: request s with done[s] != 0 pushes its ceil(ctx_len[s] / 16) pages onto the stack,
 * the last page first, requests in order (the order of hs_kv_free); their block table entries become -1 and ctx_len[s] becomes 0.
 * No page of theirs is another row's, too: rows that share pages are ended by hs_op_fork_pages (horizonserve_beams.h).
 * The lengths, the block tables and the stack stay as they were (entries of free_list behind the stack's top apart), with the status
 *     INVALID_ARG      a negative length or one beyond the block table row, or more pages than the stack has room for
 *     BAD_BLOCK_TABLE  one of the pages is outside 0 .. num_pages - 1
 */
typedef struct {
  int32_t n_seqs, max_pages_per_seq, num_pages;
  const int32_t *done;    /* device [n_seqs] */
  int32_t *ctx_len;       /* device [n_seqs] */
  int32_t *block_tables;  /* device [n_seqs, max_pages_per_seq] */
  int32_t *free_list;     /* device [num_pages] */
  int32_t *free_count;    /* device [1] */
  void *workspace;
  int32_t *status;
} hs_release_pages_t;
hs_status_t hs_op_release_pages(const hs_release_pages_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * cos / sin of rotary positions: table[p][i] = (magnitude cos(p f_i), magnitude sin(p f_i)) for p in 0 .. max_position - 1 and the
 * pairs i in 0 .. rotary_dim / 2 - 1, formed in 64 bits and rounded once to fp32.  With w_i = base^(-2 i / rotary_dim):
 *     HS_ROPE_PLAIN      f_i = w_i
 *     HS_ROPE_LINEAR     f_i = w_i / factor (positions interpolated)
 *     HS_ROPE_BASE       f_i = w'_i, from the base times factor^(rotary_dim / (rotary_dim - 2))
 *     HS_ROPE_BY_PARTS   f_i = k_i w_i + (1 - k_i) w_i / factor, k_i = clamp((n_i - turns_slow) / (turns_fast - turns_slow), 0, 1)
 *                        with n_i = trained_positions w_i / 2 pi, the turns of pair i over the trained context: pairs that turn
 *                        often are kept, slow ones are stretched
 * magnitude multiplies both (1 when the attention's scale is not changed with the context).
 */
#define HS_ROPE_PLAIN 0
#define HS_ROPE_LINEAR 1
#define HS_ROPE_BASE 2
#define HS_ROPE_BY_PARTS 3
typedef struct {
  int32_t max_position, rotary_dim; /* rotary_dim: a multiple of 16, 16 .. 256 */
  int32_t scaling;                  /* HS_ROPE_* */
  int32_t trained_positions;        /* BY_PARTS: >= 1 */
  double base, factor;              /* > 0; factor is not read by PLAIN */
  double turns_slow, turns_fast;    /* BY_PARTS: turns_fast > turns_slow */
  double magnitude;                 /* > 0 */
  float *table;                     /* device fp32 [max_position, rotary_dim / 2, 2], 16-byte aligned */
} hs_rope_table_t;
hs_status_t hs_op_rope_table(const hs_rope_table_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Rotates the first rotary_dim coordinates of every head of q and k by the token's position and stores q, and k and v in the paged
 * cache.  A pair (x, y) becomes (x c - y s, x s + y c); pair i is coordinates (i, i + rotary_dim / 2), or (2 i, 2 i + 1) when
 * interleaved.  Coordinates from rotary_dim on are copied.  Arithmetic in fp32, one rounding to the cache's type.
 * A token with tok_slot < 0 (a row that pads a captured step) is not stored in the cache.  A token whose position is outside
 * 0 .. max_position - 1 gets a q row of zeros and is not stored; where its slot is >= 0, and for a slot beyond the pool, the status
 * is INVALID_ARG.  Two tokens of a call must not share a slot.
 * head_dim: a multiple of 16, 16 .. 256; rotary_dim: a multiple of 16, 16 .. head_dim.  q, k, v and q_out rows and the row strides
 * are 16-byte aligned; kv_pool is 256-byte aligned.  q_out may be q where the types agree.
 */
typedef struct {
  int32_t n_tokens, n_q_heads, n_kv_heads, head_dim, rotary_dim, interleaved;
  int32_t src_type;                       /* HS_TYPE_* of q, k, v */
  int32_t cache_type;                     /* HS_TYPE_BF16 or HS_TYPE_F16: q_out and the pool */
  const void *q, *k, *v;                  /* device [n_tokens] rows of heads, heads contiguous */
  int64_t q_stride, k_stride, v_stride;   /* elements between rows */
  const int32_t *tok_pos, *tok_slot;      /* device [n_tokens] */
  const float *table;                     /* hs_op_rope_table's, [max_position, rotary_dim / 2, 2] */
  int32_t max_position;
  int32_t n_layers, layer, num_pages;     /* of the pool */
  void *q_out;                            /* device [n_tokens] rows of n_q_heads * head_dim */
  int64_t q_out_stride;
  void *kv_pool;
  int32_t *status;
} hs_rope_cache_t;
hs_status_t hs_op_rope_cache(const hs_rope_cache_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Attention of a step's tokens over the paged cache.  Token row t of sequence s (tok_begin[s] <= t < tok_begin[s + 1]; without
 * tok_begin, sequence s has the one row s) sits at position p = kv_len[s] - (tok_begin[s + 1] - t) and sees key j < kv_len[s] when
 *     j <= p and (window = 0 or p - j < window),   or   j < prefix_len[s]
 * -- causal, within a sliding window if there is one, and a prefix (an image, a system prompt, sinks) that every token sees.
 * For query head h, which reads KV head h / (n_q_heads / n_kv_heads),
 *     x_j = scale * q . k_j,   x_j = cap * tanh(x_j / cap) if cap > 0,   x_j -= slopes[h] * |p - j| if slopes are given,
 *     o = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)   (natural logarithm).
 * A row that sees no key gives o = 0 and lse = -infinity.  Scores, maxima, sums and o are held in fp32; the softmax weights are
 * rounded to the cache's type for the product with v (relative to a maximum, before they are divided by their sum).
 * What the cache holds at keys that no row of the call sees may be anything.  A key that some rows of a chunk see and others do not has a finite v: an infinity or
 * NaN there may reach its neighbours.
 * max_q_len: no sequence has more rows in this call (a captured loop's bound).  1 selects the form for single tokens; any other takes tiles of 128 rows of heads and
 * tokens, for sequences with one row too, so a step of prompt chunks and many single tokens is better given as two calls, one for each.  The work is planned on
 * the device from the lengths; where there is little of it, it is divided along the cache, and joined in an order that does not depend on the budget.
 * Only pages that hold a key some row sees are looked up, so block table entries that a window has left behind may be anything.
 * Status INVALID_ARG: tok_begin that falls, leaves 0 .. n_tokens or gives a sequence more than max_q_len rows; none of the sequence's rows
 * are computed.  Status BAD_BLOCK_TABLE: a page id outside the pool, or a kv_len that is negative or beyond the block table row (or 2^31 - 64);
 * nothing outside the pool is read, and the sequence's rows are not defined.
 * head_dim 64 or 128; n_q_heads a multiple of n_kv_heads, at most 1024; scale (of either sign, or 0) and cap below 1e30, cap and window >= 0.  q and o rows 16-byte aligned,
 * strides multiples of 8; kv_pool 256-byte aligned.  n_seqs <= HS_DEVICE_MAX_SEQS, n_seqs * max_pages_per_seq at most 2^27; below 2^31: that times
 * n_q_heads, n_tokens * n_q_heads, and the pool's rows (n_layers * 2 * num_pages * n_kv_heads * 16).
 */
typedef struct {
  int32_t n_seqs, n_tokens;               /* n_tokens: rows of q, o and lse (at least tok_begin[n_seqs]) */
  int32_t max_q_len;
  int32_t n_q_heads, n_kv_heads, head_dim;
  int32_t type;                           /* HS_TYPE_BF16 or HS_TYPE_F16: q, o and the pool */
  int32_t n_layers, layer, num_pages, max_pages_per_seq;
  const void *q;                          /* device rows of n_q_heads * head_dim */
  int64_t q_stride;
  const void *kv_pool;
  const int32_t *block_tables;            /* device [n_seqs, max_pages_per_seq] */
  const int32_t *kv_len;                  /* device [n_seqs]: keys with the step's own */
  const int32_t *tok_begin;               /* device [n_seqs + 1]; may be NULL when max_q_len is 1 */
  const int32_t *prefix_len;              /* device [n_seqs], or NULL */
  const float *slopes;                    /* device [n_q_heads], or NULL */
  float scale, cap;
  int32_t window;
  void *o;                                /* device rows of n_q_heads * head_dim */
  int64_t o_stride;
  float *lse;                             /* device [n_tokens, n_q_heads], or NULL */
  void *workspace;
  int32_t *status;
} hs_paged_attention_t;
hs_status_t hs_op_paged_attention(const hs_paged_attention_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Of each logit row x with l_v = scale * x_v and L = log sum_v exp(l_v):
 *     logprob = l_target - L          entropy = L - sum_v exp(l_v - L) l_v          rank = number of v with x_v > x_target
 *     top_ids[i], top_logprobs[i] = the i-th largest x_v's index, ties to the lowest index, and its l_v - L
 * A negative target: logprob 0, rank -1.  A target >= vocab: the same, and status INVALID_ARG.  Entries of -infinity (masked
 * tokens) count as probability 0; a row of nothing else has L = -infinity, and its logprobs are -infinity and its entropy 0.
 * A row that holds NaN or +infinity has NaN for L, logprob and entropy; which alternatives it names is not defined (ids -1 .. vocab - 1); its rank is as above, and
 * NaN is above nothing and has nothing above it.
 * Logits of any row stride and alignment of their type; sums in fp32.  n_rows * (vocab / 1024 + 2) below 2^31.
 * With alternatives, rows whose first 64 KB are -infinity (a vocabulary masked down to its upper end), rows that rise from end to end and rows of
 * nothing but NaN are slow: one warp looks for theirs, 12 to 22 ns an element.  A call of such rows takes 20 to 170 times as long.
 */
typedef struct {
  int32_t n_rows, vocab;       /* n_rows >= 1, 1 <= vocab < 2^30 */
  int32_t type;                /* HS_TYPE_* */
  int32_t n_top;               /* 0 .. min(HS_MAX_ALTERNATIVES, vocab) */
  const void *logits;          /* device [n_rows, vocab], rows row_stride elements apart */
  int64_t row_stride;
  const int32_t *targets;      /* device [n_rows] */
  float scale;                 /* > 0: the inverse temperature */
  float *logprob, *entropy;    /* device [n_rows]; entropy may be NULL */
  int32_t *rank;               /* device [n_rows], or NULL */
  int32_t *top_ids;            /* device [n_rows, n_top] */
  float *top_logprobs;         /* device [n_rows, n_top] */
  void *workspace;
  int32_t *status;
} hs_token_logprobs_t;
hs_status_t hs_op_token_logprobs(const hs_token_logprobs_t *a, int32_t sm_budget, void *cuda_stream);

#if defined(__GNUC__)
#pragma GCC visibility pop
#endif
#ifdef __cplusplus
}
#endif
#endif /* HORIZONSERVE_DEVICE_H_ */
