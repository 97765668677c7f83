/*
 * wt_serve — one step of many requests over one set of weights.  C ABI.
 *
 * wt_pass (wt.h) streams a checkpoint's matrices for up to 16 activation columns.  A program that
 * answers several requests with them needs four more things beside that pass, every step:
 *
 *   wt_adapt   each request's low-rank adapter beside a projection all requests share;
 *   wt_attend  attention over a prefix that all requests share, read once for all of them, and
 *              over each request's own paged cache;
 *   wt_probs   fp32 logits (wt_pass's y over the head) to probabilities at a temperature;
 *   wt_verify  drafted tokens against the target's probabilities, from given random numbers.
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
 * weights p enter the second product rounded to the caches' type.
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
