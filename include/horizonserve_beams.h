/*
 * horizonserve_beams.h -- operators of requests that continue one prompt in several ways (beam search, parallel samples, one
 * system prompt in front of many requests), beside those of horizonserve_device.h.
 *
 * Rows of block tables may share pages here.  shares[page] counts the holders of a page beyond the first, 0 for a page of one row and for a
 * free one, so hs_op_step_tables, whose new pages have one holder, needs no change.  A page that is not full has one holder: the
 * rows that append to it never meet.  Rows that share pages are ended by hs_op_fork_pages (parent -1).  hs_op_release_pages knows no holders and gives all pages of
 * a row to the stack, those of rows that go on and those that another row gives back among them: it is for rows whose pages have one holder each.
 *     hs_op_beam_select       the best continuations of every request over its beams and the vocabulary
 *     hs_op_fork_pages        rows continue other rows: shared pages counted, partly filled ones listed to be copied, dropped ones freed
 *     hs_op_copy_pages        the keys and values of listed pages, in every layer
 *     hs_op_compact_pages     pages moved below a bound, so that the pool's upper end is free
 *     hs_op_shared_attention  one new token per sequence over the paged cache; what a group of sequences shares is read once
 * A beam step is step_tables -> layers with rope_cache and shared_attention -> head -> beam_select -> fork_pages -> copy_pages.  The paper has
 * no counterpart: it keeps its runtime's KV management and model execution (Sec. 5).
 *
 * Conventions, workspace and status are those of horizonserve_device.h.
 */
#ifndef HORIZONSERVE_BEAMS_H_
#define HORIZONSERVE_BEAMS_H_

#include "horizonserve_device.h"

#ifdef __cplusplus
extern "C" {
#endif
#if defined(__GNUC__)
#pragma GCC visibility push(default)
#endif

#define HS_MAX_BEAMS 32           /* beams of a request, and continuations that a call gives it */
#define HS_BEAMS_MAX_PAGES (1 << 24)   /* pages of a pool in hs_op_fork_pages */
#define HS_COMPACT_MAX_PAGES (1 << 21) /* pages of a pool in hs_op_compact_pages */
#define HS_SHARED_MAX_SEQS 2048        /* sequences of a call of hs_op_shared_attention */

/*
 * Request r has beams b in 0 .. n_beams - 1 with accumulated log probability S_b = scores[r][b] and the logit row x = logits[r n_beams + b].
 * A beam that is not done continues with every token v,  s = S_b + scale x_v - L,  L = log sum_v exp(scale x_v);  one that is done (done != 0) has one
 * continuation, itself:  s = S_b,  v = end_token.  Continuations are ranked by weight[r][b] s (by s without weights), the largest first,
 * ties to the lower beam, then to the larger logit (a score far from zero swallows their differences) and then to the lower token, and the first n_out of them are written:
 *     out_score = s,   out_parent = r n_beams + b,   out_token = v,   out_done = whether the beam was done or v is end_token
 * A weight that is not above zero gives its beam no continuation, with the status INVALID_ARG; a call of such weights is done otherwise.
 * A weighted score of -infinity or NaN is no continuation: tokens and beams at -infinity are left out, and so is a beam whose row holds NaN or +infinity or
 * nothing above -infinity.  Where there are fewer than n_out, the rest have score -infinity, parent and token -1 and done 0.
 * A finite score or L that fp32 does not hold is written as its largest number of that sign.
 * lse[r n_beams + b] = L (0 for a beam that is done, whose logits are not read; NaN where the row holds NaN or +infinity).
 * Logits of any row stride and alignment of their type.  Exponentials in fp32, sums of a few of them too, and what is ranked in 64 bits from there on: L is within 2.5e-6 of
 * the exact one (1e-7 as a rule), and the order is that of scores as near as that; equal logits of a beam are ranked by their tokens.
 * Outputs overlap no inputs.  n_requests 1 .. HS_DEVICE_MAX_SEQS, n_requests * n_beams at most 65536.
 */
typedef struct {
  int32_t n_requests, n_beams, vocab; /* n_beams 1 .. HS_MAX_BEAMS, 1 <= vocab < 2^30 */
  int32_t type;                       /* HS_TYPE_* */
  int32_t n_out;                      /* 1 .. HS_MAX_BEAMS */
  int32_t end_token;                  /* any number; one outside the vocabulary ends no beam */
  const void *logits;                 /* device [n_requests * n_beams, vocab], rows row_stride elements apart */
  int64_t row_stride;
  const float *scores;                /* device [n_requests, n_beams] */
  const int32_t *done;                /* device [n_requests, n_beams], or NULL */
  const float *weight;                /* device [n_requests, n_beams], above zero, or NULL */
  float scale;                        /* > 0: the inverse temperature */
  float *out_score;                   /* device [n_requests, n_out] */
  int32_t *out_parent, *out_token;    /* device [n_requests, n_out] */
  int32_t *out_done;                  /* device [n_requests, n_out], or NULL */
  float *lse;                         /* device [n_requests * n_beams], or NULL */
  void *workspace;
  int32_t *status;
} hs_beam_select_t;
hs_status_t hs_op_beam_select(const hs_beam_select_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Row i of the block tables becomes a continuation of what row parent[i] held before the call, or ends (parent -1: no tokens).  A row may be continued
 * by none, one or several rows, itself among them.  Of a parent's ceil(ctx_len / 16) pages the full ones are shared by all its successors.  A last page that
 * is not full stays with the first successor (the lowest row); every other one, in row order, pops a page off the stack for it and gets an entry in the copy
 * list:  copy_src[i] -> copy_dst[i], its first copy_len[i] = ctx_len % 16 tokens (hs_op_copy_pages).  Rows without a copy have -1, -1, 0.
 * Then ctx_len[i] = ctx_len[parent[i]], entries that a row no longer owns are -1, and the pages that no row holds any more go onto the stack in rising
 * order.  Block table entries behind a row's pages, old and new, are left alone.
 * Rows outside the call may hold pages too, each counted in shares.  Two rows of a call that are continued must not share a page that is not full.
 * A call that cannot be done changes nothing but the copy list, which is empty, with the status
 *     OUT_OF_PAGES     the stack holds fewer pages than the copies need
 *     INVALID_ARG      a parent outside -1 .. n_rows - 1, a length that is negative or beyond the block table row, or free_count outside 0 .. num_pages
 * A page id outside 0 .. num_pages - 1, popped or owned, gives the status BAD_BLOCK_TABLE: it is neither counted, copied nor freed; the call is done otherwise.
 * n_rows 1 .. HS_DEVICE_MAX_SEQS, n_rows * max_pages_per_seq at most 2^27, num_pages at most HS_BEAMS_MAX_PAGES.
 */
typedef struct {
  int32_t n_rows, max_pages_per_seq, num_pages;
  const int32_t *parent;   /* device [n_rows] */
  int32_t *ctx_len;        /* device [n_rows] */
  int32_t *block_tables;   /* device [n_rows, max_pages_per_seq] */
  int32_t *shares;         /* device [num_pages] */
  int32_t *free_list;      /* device [num_pages] */
  int32_t *free_count;     /* device [1] */
  int32_t *copy_src, *copy_dst, *copy_len; /* device [n_rows] */
  void *workspace;
  int32_t *status;
} hs_fork_pages_t;
hs_status_t hs_op_fork_pages(const hs_fork_pages_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Copies the keys and values of page src[i] to page dst[i] in every layer: all 16 tokens, or the first length[i] of them (0 .. 16; others of dst stay as they
 * are).  Entries with src -1 or dst -1 are skipped.  A page id outside -1 .. num_pages - 1 or a length outside 0 .. 16 is skipped too, with the status
 * BAD_BLOCK_TABLE or INVALID_ARG.  No page is dst twice, or both src and dst.
 * head_dim a multiple of 8, at most 256; n_copies at most 2^21, n_copies * n_layers * 2 * n_kv_heads below 2^31; kv_pool 256-byte aligned.
 */
typedef struct {
  int32_t n_copies;
  int32_t type;                          /* HS_TYPE_BF16 or HS_TYPE_F16 */
  int32_t n_layers, num_pages, n_kv_heads, head_dim; /* of the pool */
  const int32_t *src, *dst;              /* device [n_copies] */
  const int32_t *length;                 /* device [n_copies], or NULL: whole pages */
  void *kv_pool;
  int32_t *status;
} hs_copy_pages_t;
hs_status_t hs_op_copy_pages(const hs_copy_pages_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Makes pages n_keep .. num_pages - 1 free, for a pool that is to be smaller or whose upper end another stage is to have.  Pages that are not on the stack are in use:
 * the k-th of them from n_keep up (in rising order) moves to the k-th free page below n_keep (in rising order).  copy_src[k], copy_dst[k] list the moves for
 * hs_op_copy_pages, -1 behind the last one.  The first ceil(ctx_len / 16) entries of every block table row follow; a holder that is not a row of the call
 * follows the copy list.  shares moves with the pages.  The stack is left with the same number of pages, the highest first: new ones come from the pool's lower end, and
 * its first num_pages - n_keep entries are the upper end, which a caller may take away.
 * A call that cannot be done changes nothing but the copy list, which is empty, with the status
 *     OUT_OF_PAGES     fewer free pages below n_keep than moves
 *     INVALID_ARG      more moves than max_copies, a negative length or one beyond the block table row, free_count outside 0 .. num_pages, or a stack that
 *                      holds a page twice or one outside the pool
 * A block table entry outside the pool, or one from n_keep up that is on the stack, stays as it is, with the status BAD_BLOCK_TABLE.
 * n_rows 1 .. HS_DEVICE_MAX_SEQS, n_rows * max_pages_per_seq at most 2^27, num_pages at most HS_COMPACT_MAX_PAGES, 0 <= n_keep <= num_pages.
 */
typedef struct {
  int32_t n_rows, max_pages_per_seq, num_pages, n_keep, max_copies;
  const int32_t *ctx_len;  /* device [n_rows] */
  int32_t *block_tables;   /* device [n_rows, max_pages_per_seq] */
  int32_t *shares;         /* device [num_pages] */
  int32_t *free_list;      /* device [num_pages] */
  const int32_t *free_count; /* device [1] */
  int32_t *copy_src, *copy_dst; /* device [max_copies] */
  void *workspace;
  int32_t *status;
} hs_compact_pages_t;
hs_status_t hs_op_compact_pages(const hs_compact_pages_t *a, int32_t sm_budget, void *cuda_stream);

/*
 * Attention of one new token per sequence, as hs_op_paged_attention with max_q_len 1: row s of q is sequence s, at position p = kv_len[s] - 1, and sees all
 * keys j < kv_len[s],
 *     x_j = scale * q . k_j,   x_j = cap * tanh(x_j / cap) if cap > 0,   x_j -= slopes[h] * (p - j) if slopes are given,
 *     o = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)   (natural logarithm).
 * Group g is sequences group_begin[g] .. group_begin[g + 1] - 1.  Its shared_len[g] first keys are the same for all of them: counted down to whole pages, and to the
 * shortest of its sequences that have keys at all, they are read through the block table row of the first of those, once for the group.  Where the rows' tables or the pages
 * differ there, the result is that of the pages read.  A sequence outside all groups is not computed, its rows are left as they were; one without keys gives o = 0, lse = -infinity.
 * Scores, maxima, sums and o are held in fp32; the softmax weights are rounded to the cache's type for the product with v, before they are divided by their
 * sum.  What the cache holds behind a sequence's keys may be anything, and an infinity or NaN at a key reaches the rows that see it, and no others.  (Rows of one tile with a row that
 * sees an infinite or NaN v are worked out by themselves, with unrounded weights: such a call takes milliseconds behind a long prompt.)
 * It pays where the sequences' keys and values, counted one by one, come to some 200 MB; below that hs_op_paged_attention, with max_q_len 1, takes down to half the time.
 * Work is planned on the device from the lengths, divided along the keys, and joined in an order that does not depend on the budget.  Where it is divided depends on the
 * lengths of all sequences of the call: next to others, a sequence's o and lse may differ in the last bits, within the roundings above.
 * Status INVALID_ARG: group_begin that falls or leaves 0 .. n_seqs, a negative shared_len; nothing is computed.  Status BAD_BLOCK_TABLE: a page id outside
 * the pool, or a kv_len that is negative or beyond the block table row (or 2^31 - 64); nothing outside the pool is read, and the rows of the group are not defined.
 * head_dim 64 or 128; n_q_heads a multiple of n_kv_heads, at most 1024; scale and cap as in hs_op_paged_attention.  q and o rows 16-byte aligned, strides multiples
 * of 8; kv_pool 256-byte aligned.  n_groups <= n_seqs <= HS_SHARED_MAX_SEQS, n_seqs * max_pages_per_seq at most 2^26; below 2^30: that times n_q_heads; below 2^31: the pool's
 * rows (n_layers * 2 * num_pages * n_kv_heads * 16).
 */
typedef struct {
  int32_t n_seqs, n_groups, n_q_heads, n_kv_heads, head_dim;
  int32_t type;                           /* HS_TYPE_BF16 or HS_TYPE_F16: q, o and the pool */
  int32_t n_layers, layer, num_pages, max_pages_per_seq;
  const void *q;                          /* device [n_seqs] rows of n_q_heads * head_dim */
  int64_t q_stride;
  const void *kv_pool;
  const int32_t *block_tables;            /* device [n_seqs, max_pages_per_seq] */
  const int32_t *kv_len;                  /* device [n_seqs] */
  const int32_t *group_begin;             /* device [n_groups + 1] */
  const int32_t *shared_len;              /* device [n_groups] */
  const float *slopes;                    /* device [n_q_heads], or NULL */
  float scale, cap;
  void *o;                                /* device [n_seqs] rows of n_q_heads * head_dim */
  int64_t o_stride;
  float *lse;                             /* device [n_seqs, n_q_heads], or NULL */
  void *workspace;
  int32_t *status;
} hs_shared_attention_t;
hs_status_t hs_op_shared_attention(const hs_shared_attention_t *a, int32_t sm_budget, void *cuda_stream);

#if defined(__GNUC__)
#pragma GCC visibility pop
#endif
#ifdef __cplusplus
}
#endif
#endif /* HORIZONSERVE_BEAMS_H_ */
