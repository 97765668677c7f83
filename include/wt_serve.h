/*
 * wt_serve — one step of many requests over one set of weights.  C ABI.
 *
 * wt_pass (wt.h) streams a checkpoint's matrices for up to 16 activation columns.  A program that
 * answers several requests with them needs seven more things beside that pass, every step:
 *
 *   wt_adapt     each request's low-rank adapter beside a projection all requests share;
 *   wt_place     the projections' rows to normed and rotated queries, and keys and values in their pages;
 *   wt_attend    attention over a prefix that all requests share, read once for all of them, and
 *                over each request's own paged cache;
 *   wt_cross     attention of each request's tokens to a memory of its own, as an encoder's states;
 *   wt_probs     fp32 logits (wt_pass's y over the head) to probabilities at a temperature;
 *   wt_logprobs  log probabilities of given tokens, entropy and the likeliest tokens of such logits;
 *   wt_verify    drafted tokens against the target's probabilities, from given random numbers.
 *
 * Conventions are those of wt.h: int status codes and wt_last_error, void* streams, caller-owned
 * device memory, no C++ exception across the boundary.  Besides:
 *   - A handle supplies the device, the status word and the workspaces; wt_open with no path gives
 *     one.  A call enqueues its kernels on `stream` and returns; nothing waits on the host for the
 *     device (a call larger than those before it on its stream allocates).
 *   - Workspaces belong to the handle and stay until wt_close.  Each stream has its own; from the
 *     ninth stream on a new one takes over those of a stream whose calls have completed.  A call
 *     captured into a CUDA graph takes a workspace of its own; every replay must complete before
 *     wt_close, and two replays of one graph must not overlap.  No warm-up call is needed before a
 *     capture.
 *   - wt_close waits for the last call on each stream, and for nothing else on the device.  Calls
 *     and wt_close may be made while another thread captures.
 *   - Descriptors are read during the call and not kept.
 *   - Lengths, slots, page numbers and tokens that lie in device memory cannot be checked on the
 *     host.  Where one contradicts its descriptor, the kernel clamps it (an offset, a length, a
 *     rank) or treats its element as absent (a page, a slot, a drafted token), reads and writes
 *     nothing outside the descriptor's buffers, and records WT_EINVAL in the handle's status word
 *     (wt_device_status) if nothing was recorded there before.
 *   - Results are deterministic: no floating-point atomics, and no result depends on timing.  A
 *     token's last bits may depend on what else a call holds: how its sums are split over CTAs
 *     follows the numbers of tokens, slots and keys.  (wt_verify's tokens never do.)
 */
#ifndef WT_SERVE_H_
#define WT_SERVE_H_

#include "wt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- wt_adapt -------------------------------------------------------------------------------
 * y[t] = base[t] + scale[s] * B_s (A_s x[t]),   s = slot[t],  t < T
 *
 * A token whose slot is negative has no adapter: y[t] = base[t].  A is [S, R, K] and B is
 * [S, M, R], row-major within a slot, as checkpoints store the two factors ([out, in]); slots lie
 * a_slot and b_slot elements apart.  A slot of rank[s] < R uses the first rank[s] rows of A and
 * columns of B only; what lies in the others is never used (NaN there is harmless).  x is bf16 or
 * f16, as are A and B; base and y are fp32, as wt_pass leaves them.  A x is summed in fp32 and
 * enters the second product with 22 bits or more (of the token's largest number), which is summed in
 * fp32.
 * base may be y itself (then tokens without adapter cost nothing).  base NULL stands for zeros.
 *
 * All descriptors of a call share one launch per 8 of them (three launches from 256 tokens on).
 * No y may overlap what its own or another descriptor reads, or another's y; a call refuses that where
 * the two share a launch.  (Rows count, not the bytes between them: columns of one buffer are fine.)
 * T, K and M go up to 2^30, R up to 128, at any element alignment; rows that lie on 16-byte boundaries
 * load faster. */
#define WT_ADAPT_MAX_RANK 128
#define WT_ADAPT_MAX_SLOTS 4096
typedef struct {
  const void *x;        /* [T, K], row pitch ldx elements */
  const float *base;    /* [T, M], row pitch ldbase; NULL: zeros; may equal y (with ldbase == ldy) */
  float *y;             /* [T, M], row pitch ldy */
  const int32_t *slot;  /* [T]; < 0: no adapter */
  const void *A;        /* [S, R, K] */
  const void *B;        /* [S, M, R] */
  const int32_t *rank;  /* [S], or NULL: R for every slot */
  const float *scale;   /* [S], or NULL: 1 */
  int64_t ldx, ldbase, ldy;
  int64_t a_slot, b_slot; /* elements from one slot to the next: >= R K, >= M R */
  int32_t dtype;        /* WT_BF16 or WT_F16 */
  int32_t T, K, M, S, R;
} wt_adapt_desc;

/* Errors: WT_EINVAL (NULL, a size outside its range, a pitch below its row, a buffer that runs past
 * its device allocation, y inside a mapping), WT_ENOTSUP (dtype, host-only handle), WT_ECUDA. */
int wt_adapt(wt_handle *h, const wt_adapt_desc *d, size_t n, void *stream);

/* ---- wt_place -------------------------------------------------------------------------------
 * What stands between the projections and wt_attend, in one pass over their rows.  For token i of
 * request b (row t = begin[b] + i), each head of q and k goes
 *
 *   y  = x * w / sqrt(mean(x^2) + eps)          where q_norm (k_norm) gives w, over the whole head
 *   (y0, y1) <- (y0 cos a - y1 sin a, y1 cos a + y0 sin a)   for pair j of the first rot_dim elements
 *
 * and is rounded once: q to q_out[t], k and (unchanged) v to the caches' row of the token's place
 * len[b] - n_b + i, which wt_attend finds again: row place % page of page table[b, place / page].
 * Any of q, k and v may be NULL (with its output): then it is not looked at.  q alone needs no pages, and
 * v alone no turns and no pos.
 *
 * Pair j is elements j and j + rot_dim / 2, or with WT_PLACE_NEIGHBOURS 2j and 2j + 1.  Its angle is
 * pos * 2 pi * turns[j] / 2^64: turns[j] holds the turns that a position adds, modulo one, as a fraction
 * in 64 bits, so the angle is exact modulo a turn at any position (2^64 f / 2 pi for f radians a position;
 * serving.turns).  pos is the token's own position on axis[j] of the axes of `pos` (time, height, width),
 * or without `pos` first_pos + place.
 *
 * The rows are fp32 (as wt_pass and wt_adapt leave them) or of the caches' type; sums and products are
 * fp32.  Rows of tokens that no request holds are left as they are; without `begin` (q alone, with pos or
 * without rotation) every row counts.  A token whose place is negative (more new tokens than len) or whose
 * page is out of range is not cached, and WT_EINVAL recorded; its query is made all the same.  Where two
 * new tokens share a place (one page in the tables of two requests) either may stand there.
 *
 * head_dim is a multiple of 8 up to 256, rot_dim one up to head_dim; heads and kv_heads go up to 65536;
 * n_tokens, max_len and first_pos up to 2^30.  Pointers to rows and pages lie on 16-byte boundaries and
 * their strides are multiples of 8 elements.  q_out may be q (of one type, at its pitch); otherwise no
 * output may overlap an input or another output, as rows of tokens. */
#define WT_PLACE_MAX_DIM 256
#define WT_PLACE_MAX_AXES 8
#define WT_PLACE_NEIGHBOURS 1 /* a flag */
typedef struct {
  const void *q;            /* [n_tokens, heads, head_dim], token pitch q_stride elements */
  const void *k, *v;        /* [n_tokens, kv_heads, head_dim], token pitches k_stride and v_stride */
  void *q_out;              /* [n_tokens, heads, head_dim], token pitch out_stride */
  void *k_pages, *v_pages;  /* [n_pages, page, kv_heads, head_dim], dense */
  const void *q_norm, *k_norm; /* [head_dim] of norm_dtype; NULL: no norm */
  const int32_t *begin;     /* [n_req + 1]: first token of each request, ascending, begin[n_req] <= n_tokens */
  const int32_t *table;     /* [n_req, pages of max_len keys] page numbers, row pitch table_stride */
  const int32_t *len;       /* [n_req] own keys, the new tokens' included; <= max_len */
  const uint64_t *turns;    /* [rot_dim / 2] */
  const int32_t *pos;       /* [n_tokens, axes], row pitch pos_stride, or NULL */
  int64_t q_stride, k_stride, v_stride, out_stride, table_stride, pos_stride;
  int32_t in_dtype;         /* of q, k, v: WT_F32 or dtype */
  int32_t dtype;            /* WT_BF16 or WT_F16 */
  int32_t norm_dtype;       /* WT_F32, WT_BF16 or WT_F16 */
  int32_t n_req, n_tokens, heads, kv_heads, head_dim, rot_dim, axes;
  int32_t page, n_pages, max_len, first_pos, flags;
  float eps;                /* >= 0 */
  uint8_t axis[WT_PLACE_MAX_DIM / 2]; /* of each pair, < axes */
} wt_place_desc;

/* Errors: WT_EINVAL (NULL, sizes, alignment, strides, an output inside a mapping or over an input, a buffer
 * that runs past its device allocation), WT_ENOTSUP (dtype, head_dim, host-only handle), WT_ECUDA. */
int wt_place(wt_handle *h, const wt_place_desc *d, void *stream);

/* ---- wt_attend ------------------------------------------------------------------------------
 * Token i of request b (row t = begin[b] + i of q, i < n_b = begin[b + 1] - begin[b]) attends to the
 * whole shared prefix and to its request's own keys 0 .. len[b] - n_b + i (its own key included: the
 * new tokens' keys are the last n_b of the cache):
 *
 *   out[t, h] = sum_j p_j v_j,   p = softmax_j(scale * q[t, h] . k_j),   kv head h / (heads / kv_heads)
 *
 * A token that sees no key at all gets zeros, and so does one all of whose scores are -infinity: such
 * a key has no weight.  A NaN in its query or in a key that it sees makes a token's head NaN, and a
 * value that is not finite makes its column so, however small its weight.  Own keys live in pages: key
 * j of request b is row j % page of page table[b, j / page].  Rows of a page past len[b] are never
 * used, and a later token's key and value never reach an earlier one (NaN and infinity there are
 * harmless).  q, caches and out are bf16 or f16; scores, softmax statistics and sums are fp32, and the
 * weights p enter the second product rounded to the caches' type.  That product's sums are cut off where they
 * grow: with many rows, results of values of one sign fall short by some 4e-9 of themselves for each key of the
 * prefix, by two roundings of f16 for 2^18 keys.
 *
 * head_dim is a multiple of 8 up to 128; heads a multiple of kv_heads, heads / kv_heads <= 128; n_req
 * is below 65536, n_tokens, prefix_len and max_len go up to 2^30, n_tokens * heads to 2^31 - 1.
 * Pointers lie on 16-byte boundaries and strides are multiples of 8 elements.  prefix_len 0 or
 * max_len 0 leave that part out (its pointers may be NULL).  out may be q itself (at its pitch);
 * otherwise it must not overlap any input, as rows of tokens. */
typedef struct {
  const void *q;            /* [n_tokens, heads, head_dim], token pitch q_stride elements */
  void *out;                /* [n_tokens, heads, head_dim], token pitch out_stride */
  const int32_t *begin;     /* [n_req + 1]: first token of each request, ascending, begin[n_req] <= n_tokens */
  const void *prefix_k;     /* [prefix_len, kv_heads, head_dim], key pitch prefix_stride, head pitch prefix_head */
  const void *prefix_v;     /* the same pitches */
  const void *k_pages;      /* [n_pages, page, kv_heads, head_dim], dense */
  const void *v_pages;
  const int32_t *table;     /* [n_req, pages of max_len keys] page numbers, row pitch table_stride */
  const int32_t *len;       /* [n_req] own keys, the new tokens' included; <= max_len */
  int64_t q_stride, out_stride, prefix_stride, prefix_head, table_stride;
  int64_t prefix_len;
  int32_t dtype;            /* WT_BF16 or WT_F16 */
  int32_t n_req, n_tokens, max_new; /* max_new: no request has more new tokens */
  int32_t heads, kv_heads, head_dim;
  int32_t page, n_pages, max_len;
  float scale;
  int32_t pad;
} wt_attend_desc;

/* Errors: WT_EINVAL (NULL, sizes, alignment, strides, out inside a mapping, a buffer that runs past
 * its device allocation), WT_ENOTSUP (dtype, head_dim, host-only handle), WT_ENOMEM, WT_ECUDA. */
int wt_attend(wt_handle *h, const wt_attend_desc *d, void *stream);

/* ---- wt_cross -------------------------------------------------------------------------------
 * Token i of request b (row begin[b] + i of q) attends to its request's memory, the states
 * mem_begin[b] .. mem_begin[b] + mem_len[b] - 1 of k and v, whole (nothing is causal here):
 *
 *   out[t, h] = sum_j p_j v_j,   p = softmax_j(scale * q[t, h] . k_j),   kv head h / (heads / kv_heads)
 *
 * over the states with keep[j] != 0 (keep NULL: all).  Memories may overlap or be one; a request's tokens
 * read theirs once, so beams or drafts over one memory are best one request's tokens.  Scores and sums are
 * fp32, whatever a memory's length; weights are rounded to the memory's type, and divided by the sum of the
 * rounded ones.  A token that sees no state gets zeros, and so does one all of whose scores are -infinity.
 * NaN and infinities show as wt_attend's do; what is not in the memory, or not kept, never reaches a result,
 * whatever stands there.  Rows of tokens that no request holds are left as they are.
 *
 * Types, head sizes and limits are wt_attend's; n_mem goes up to 2^30.  out may be q itself (at its
 * pitch); otherwise it must not overlap any input, as rows of tokens. */
typedef struct {
  const void *q;            /* [n_tokens, heads, head_dim], token pitch q_stride elements */
  void *out;                /* [n_tokens, heads, head_dim], token pitch out_stride */
  const int32_t *begin;     /* [n_req + 1]: first token of each request, ascending, begin[n_req] <= n_tokens */
  const void *k;            /* [n_mem, kv_heads, head_dim], state pitch mem_stride, head pitch mem_head */
  const void *v;            /* the same pitches */
  const int32_t *mem_begin; /* [n_req] first state of each request's memory */
  const int32_t *mem_len;   /* [n_req] <= max_mem */
  const uint8_t *keep;      /* [n_mem], or NULL */
  int64_t q_stride, out_stride, mem_stride, mem_head, n_mem;
  int32_t dtype;            /* WT_BF16 or WT_F16 */
  int32_t n_req, n_tokens, max_new, max_mem; /* no request has more new tokens, no memory more states */
  int32_t heads, kv_heads, head_dim;
  float scale;
  int32_t pad;
} wt_cross_desc;

/* Errors: WT_EINVAL (NULL, sizes, alignment, strides, out inside a mapping, a buffer that runs past
 * its device allocation), WT_ENOTSUP (dtype, head_dim, host-only handle), WT_ENOMEM, WT_ECUDA. */
int wt_cross(wt_handle *h, const wt_cross_desc *d, void *stream);

/* ---- wt_probs -------------------------------------------------------------------------------
 * p[r, v] = exp((l[r, v] - m_r) / temp[r]) / sum,  m_r the row's largest logit.
 *
 * temp[r] that is not above zero draws greedily: p is 1 at the first of the row's largest logits and
 * 0 elsewhere.  A logit of -infinity has probability 0; a row of nothing else is all zeros.  NaN or
 * +infinity in a row with temp > 0 makes the row NaN; a greedy row ignores NaN.  p may be the logits
 * themselves (ldp == ldl), otherwise p must not overlap logits or temp (as rows). */
typedef struct {
  const float *logits;  /* [rows, vocab], row pitch ldl */
  float *p;             /* [rows, vocab], row pitch ldp */
  const float *temp;    /* [rows], or NULL: 1 */
  int64_t ldl, ldp;
  int32_t rows, vocab;
} wt_probs_desc;

/* Errors: WT_EINVAL, WT_ENOTSUP (host-only handle), WT_ECUDA. */
int wt_probs(wt_handle *h, const wt_probs_desc *d, void *stream);

/* ---- wt_logprobs ----------------------------------------------------------------------------
 * Of the distribution p that wt_probs gives a row, from one reading of its logits:
 *
 *   given_lp[r, i] = log p[r, given[r, i]]     (given negative: no token, 0)
 *   entropy[r]     = -sum p log p
 *   top[r, i]      the i-th largest logit's token, of equal logits the first token first; top_lp its log p
 *
 * A token of probability 0 has -infinity.  top lists no NaN and no logit of -infinity; where a row has
 * fewer others than n_top the rest is token -1 with -infinity.  A row with temp <= 0 is certain of its
 * first largest logit (0 for it, -infinity for all others, entropy 0); top still goes by the logits.  A
 * row of -infinity alone has -infinity everywhere and entropy 0; a row that wt_probs makes NaN has NaN
 * (its tokens in top are those of its largest logits).  A given token past the vocabulary counts as none,
 * and WT_EINVAL is recorded.  given, entropy and top may each be NULL.  Outputs are dense and must not
 * overlap the inputs or each other. */
#define WT_LOGPROBS_MAX_TOP 32
typedef struct {
  const float *logits;   /* [rows, vocab], row pitch ldl */
  const float *temp;     /* [rows], or NULL: 1 */
  const int32_t *given;  /* [rows, n_given], row pitch given_stride */
  float *given_lp;       /* [rows, n_given] */
  float *entropy;        /* [rows] */
  int32_t *top;          /* [rows, n_top] */
  float *top_lp;         /* [rows, n_top] */
  int64_t ldl, given_stride;
  int32_t rows, vocab, n_given, n_top;
} wt_logprobs_desc;

/* Errors: WT_EINVAL, WT_ENOTSUP (host-only handle), WT_ENOMEM, WT_ECUDA. */
int wt_logprobs(wt_handle *h, const wt_logprobs_desc *d, void *stream);

/* ---- wt_verify ------------------------------------------------------------------------------
 * Request b drafted n_b = begin[b + 1] - begin[b] tokens.  Row begin[b] + b + i of p holds the
 * target's probabilities at position i <= n_b (one row more than drafts), row begin[b] + i of q the
 * draft's.  Token i stays while
 *
 *   u[begin[b] + i] * q(token) < p(token)      (fp32, the product rounded to nearest)
 *
 * for it and every one before it; accepted[b] counts those that stay.  One token is drawn after
 * them: at a refused position from max(p - q, 0), after the last draft from p.  q NULL: the draft
 * was certain of its tokens (q is 1 there and 0 elsewhere).  tokens[b] holds the accepted tokens,
 * then the drawn one, then -1.
 *
 * The draw is exact and does not depend on how the row is split: token v weighs
 * w(v) = floor(min(x, 1) 2^40), an integer (NaN and negative x weigh 0); S is the sum, and the
 * token drawn is the first whose running sum exceeds floor(floor(u_draw 2^24) S / 2^24).  Where
 * S = 0 at a refused position (p <= q everywhere: equal up to rounding) the token is drawn from p;
 * where that has S = 0 too, it is -1.  A drafted token outside 0 .. vocab - 1 is refused.  u and
 * u_draw lie in [0, 1).  n_drafted goes up to 2^30, n_req to 2^24, max_draft to 2^20.
 * accepted and tokens must not overlap the inputs or each other. */
#define WT_VERIFY_MAX_VOCAB (1 << 18)
typedef struct {
  const float *p;          /* [n_drafted + n_req, vocab], row pitch ldp */
  const float *q;          /* [n_drafted, vocab], row pitch ldq, or NULL */
  const int32_t *drafted;  /* [n_drafted] */
  const int32_t *begin;    /* [n_req + 1], ascending, begin[n_req] <= n_drafted */
  const float *u;          /* [n_drafted] */
  const float *u_draw;     /* [n_req] */
  int32_t *accepted;       /* [n_req] */
  int32_t *tokens;         /* [n_req, max_draft + 1] */
  int64_t ldp, ldq;
  int32_t n_req, n_drafted, max_draft, vocab;
} wt_verify_desc;

/* Errors: WT_EINVAL, WT_ENOTSUP (host-only handle), WT_ECUDA. */
int wt_verify(wt_handle *h, const wt_verify_desc *d, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* WT_SERVE_H_ */
