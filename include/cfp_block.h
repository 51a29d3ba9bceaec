/*
 * cfp_block.h -- C ABI of the decoder-block operators (libcfp_block.so, gfx950).
 *
 * The plan search (cfp.h) takes the time of every block of a model under every
 * strategy.  These are operators that such blocks are made of, in the shapes that a
 * strategy leaves to one device: tokens, heads, experts or inner width divided
 * over the devices.
 *
 *   cfp_qk_norm_rope    root-mean-square norm of queries and keys for each head, with
 *                       the position rotation in the same pass; and its gradient
 *   cfp_route           routing of tokens to experts; and its gradient
 *   cfp_expert_plan     order of the assignments by expert
 *   cfp_experts         the experts' products over that order; and their gradient
 *   cfp_cache_write     keys and values of new tokens into a paged cache, quantised as they are written
 *   cfp_cache_read      the tokens of sequences back from it
 *   cfp_attend          attention of new tokens over it
 *
 * Conventions (as in cfp.h): the caller owns all memory; nothing is allocated, kept or
 * synchronised; work is enqueued on `stream` and may be captured into a graph; argument
 * errors are returned as CFP_ERR_* before any HIP call.  16-bit and 32-bit element
 * types are CFP_DT_*; sums are held in 32 bits; a result is rounded to its type once.  The
 * experts' products round operands between them as well, see there.
 * The experts' workspaces, what they keep and the attention's workspace start on 16 bytes, other workspaces on 4 (CFP_ERR_ARG);
 * tensors on their type, but a cache's pages, what cfp_cache_read writes and the result of cfp_attend on 16 bytes.
 * Results do not depend on the order in which workgroups run.  A call with no tokens
 * writes what does not depend on them (the plan's offsets, gradients of zero) and returns CFP_OK.
 */
#ifndef CFP_BLOCK_H
#define CFP_BLOCK_H

#include "cfp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CFP_DT_F32 = 0, CFP_DT_F16 = 1, CFP_DT_BF16 = 2 };

/* ---- queries and keys ---- */

#define CFP_QK_MAX_DIM 512

typedef struct {
  int64_t n_tokens;
  int32_t n_q, n_k;       /* heads of the queries and of the keys (either may be 0) */
  int32_t dim;            /* of a head, 1 <= dim <= CFP_QK_MAX_DIM */
  int32_t rot;            /* leading entries that are rotated, even, 0 <= rot <= dim */
  int32_t interleaved;    /* pairs: 0: (i, i + rot/2); 1: (2i, 2i+1) */
  int32_t dtype, wdtype;  /* of q, k and the outputs; of the gains */
  float eps;
  int64_t n_pos;          /* rows of cos and sin */
  const void *q, *k;      /* device [n_tokens][heads][dim], last dimension contiguous */
  int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride; /* in elements */
  const void *wq, *wk;    /* device [dim] gains, or NULL for ones */
  const float *cos, *sin; /* device [n_pos][rot/2] */
  const int32_t *pos;     /* device [n_tokens], or NULL: token t has position t.  A position
                             outside [0, n_pos) turns the rotated entries of its rows into NaN */
} cfp_qk_desc;

/* yq [n_tokens][n_q][dim], yk [n_tokens][n_k][dim], contiguous: each head over its
 * root mean square (sqrt(mean of squares + eps)), times the gain, with the leading `rot` entries rotated. */
int cfp_qk_norm_rope(const cfp_qk_desc *d, void *yq, void *yk, void *stream);

/* Gradients of cfp_qk_norm_rope from dyq, dyk (strides in elements; last dimension contiguous):
 * dq, dk as yq and yk; dwq, dwk [dim] float (NULL: not wanted). */
size_t cfp_qk_workspace_bytes(const cfp_qk_desc *d);
int cfp_qk_norm_rope_bwd(const cfp_qk_desc *d, const void *dyq, int64_t dyq_token_stride, int64_t dyq_head_stride,
                         const void *dyk, int64_t dyk_token_stride, int64_t dyk_head_stride, void *dq, void *dk,
                         float *dwq, float *dwk, void *ws, size_t ws_bytes, void *stream);

/* The same with positions of several axes (of an image: its row and its column): d->pos is [n_axes][n_tokens], and pair i of
 * the rotated entries takes its angle from the tables' row pos[axis[i]][t].  axis: host [rot / 2], values below
 * n_axes, read before the call returns.  A position outside the tables turns the entries of its axis into NaN. */
#define CFP_QK_MAX_AXES 4
int cfp_qk_norm_rope_axes(const cfp_qk_desc *d, const uint8_t *axis, int32_t n_axes, void *yq, void *yk, void *stream);
int cfp_qk_norm_rope_axes_bwd(const cfp_qk_desc *d, const uint8_t *axis, int32_t n_axes, const void *dyq,
                              int64_t dyq_token_stride, int64_t dyq_head_stride, const void *dyk, int64_t dyk_token_stride,
                              int64_t dyk_head_stride, void *dq, void *dk, float *dwq, float *dwk, void *ws,
                              size_t ws_bytes, void *stream);

/* ---- routing ---- */

#define CFP_ROUTE_MAX_EXPERTS 1024
#define CFP_ROUTE_MAX_K 32

enum { CFP_SCORE_SOFTMAX = 0, CFP_SCORE_SIGMOID = 1 };
enum { CFP_GROUP_MAX = 0, CFP_GROUP_TOP_TWO = 1 };

typedef struct {
  int64_t n_tokens;
  int32_t n_experts;          /* 1 .. CFP_ROUTE_MAX_EXPERTS */
  int32_t k;                  /* experts of a token, 1 .. min(n_experts, CFP_ROUTE_MAX_K) */
  int32_t score;              /* CFP_SCORE_* */
  int32_t groups, top_groups; /* equal consecutive groups, of which top_groups stay (1, 1: none) */
  int32_t group_score;        /* CFP_GROUP_*: a group's largest value, or the sum of the two largest of its scores + bias */
  int32_t renormalise;        /* weights over their sum */
  int32_t dtype;              /* of the logits */
  float scale;                /* of the weights */
  const void *logits;         /* device [n_tokens][n_experts], rows `stride` elements apart */
  int64_t stride;
  const float *bias;          /* device [n_experts], added to the scores for the selection only; or NULL */
} cfp_route_desc;

/* weight [n_tokens][k] float and index [n_tokens][k] int32: the experts with the largest
 * selection value (score + bias; without a bias the logit, whose order is the scores'), largest first, equal
 * ones by the lowest index.  A logit of -inf masks its expert: it has score 0 and is never
 * taken.  A place for which no expert is left has index -1 and weight 0.  NaN counts as the
 * least value that is not masked. */
int cfp_route(const cfp_route_desc *d, float *weight, int32_t *index, void *stream);

/* Gradient of the weights in the logits, for the experts in `index` (distinct in a row;
 * negative: none): dlogits [n_tokens][n_experts] contiguous, in the logits' type.  The bias has none. */
int cfp_route_bwd(const cfp_route_desc *d, const int32_t *index, const float *dweight, void *dlogits, void *stream);

/* ---- experts ---- */

typedef struct {
  int64_t n_tokens;
  int32_t k;
  int32_t n_experts, first; /* the experts first .. first + n_experts - 1; assignments to others are dropped */
  const int32_t *index;     /* device [n_tokens][k] */
} cfp_plan_desc;

/* Stable order of the assignments a = token * k + place by expert:
 *   offsets [n_experts + 1]   expert e has the positions offsets[e] .. offsets[e+1] - 1
 *   rows    [n_tokens * k + CFP_PLAN_PAD]  assignment at each position, -1 behind the last one kept
 *   slot    [n_tokens * k]    position of each assignment, -1 where it is dropped */
#define CFP_PLAN_PAD 16
size_t cfp_expert_plan_workspace_bytes(const cfp_plan_desc *d);
int cfp_expert_plan(const cfp_plan_desc *d, int32_t *offsets, int32_t *rows, int32_t *slot, void *ws, size_t ws_bytes,
                    void *stream);

/* Rounding between the products: silu(gate) * up, its gradient in gate and up, and weight * silu(gate) * up are the
 * next product's operands and are rounded to 8 bits (bfloat16) or 11 (float16) once; gate, up, dweight, the
 * experts' outputs before the sum over a token's experts and the rows of dx are in 32 bits.  Magnitudes between the
 * products are those of 32-bit floats for both types: float16 operands are rounded under a power of two for each
 * vector that a product sums over, so that entries within 2^28 of the vector's largest keep their 11 bits. */

#define CFP_EXPERTS_MAX_K 64
#define CFP_EXPERTS_MAX_DIM 32768

typedef struct {
  int64_t n_tokens;
  int32_t k, n_experts;
  int32_t hidden, inner;    /* 1 .. CFP_EXPERTS_MAX_DIM */
  int32_t dtype;            /* CFP_DT_F16 or CFP_DT_BF16: of x, w1, w2, y and their gradients */
  const void *x;            /* device [n_tokens][hidden], rows x_stride elements apart */
  int64_t x_stride;
  const void *w1;           /* device [n_experts][2 inner][hidden]: gate rows, then up rows */
  const void *w2;           /* device [n_experts][hidden][inner] */
  const float *weight;      /* device [n_tokens][k] */
  const int32_t *offsets, *rows, *slot; /* of cfp_expert_plan */
} cfp_experts_desc;

/* y [n_tokens][hidden]: sum over a token's assignments of weight * W2 (silu(W1g x) * (W1u x)).
 * A token without any gets zeros.  kept: what the gradient needs, cfp_experts_kept_bytes, or NULL. */
size_t cfp_experts_kept_bytes(const cfp_experts_desc *d);
size_t cfp_experts_workspace_bytes(const cfp_experts_desc *d, int32_t backward);
int cfp_experts(const cfp_experts_desc *d, void *y, void *kept, void *ws, size_t ws_bytes, void *stream);

/* Gradients from dy [n_tokens][hidden] (rows dy_stride elements apart): dx [n_tokens][hidden],
 * dw1 and dw2 as w1 and w2 (zeros for an expert without assignments), dweight [n_tokens][k] (0 where dropped). */
int cfp_experts_bwd(const cfp_experts_desc *d, const void *dy, int64_t dy_stride, const void *kept, void *dx, void *dw1,
                    void *dw2, float *dweight, void *ws, size_t ws_bytes, void *stream);

/* ---- keys and values of past tokens ---- */

/* Floats of 8 bits with 4 exponent bits, no infinities (OCP E4M3): of a cache only. */
#define CFP_DT_E4M3 3
#define CFP_CACHE_MAX_DIM 256
#define CFP_CACHE_MAX_PAGE 256
#define CFP_MAX_SEQUENCES (1 << 20)

/* Keys [n_pages][heads][page][dim] and values [n_pages][heads][dim][page]: a value's tokens lie behind each other, as
 * the product over tokens takes them.  Entries of CFP_DT_E4M3 stand for themselves times 2^(scale - 127) with a scale
 * from 1 to 254 for each token and head, [n_pages][heads][page].  Pages may lie apart; the inner dimensions are contiguous. */
typedef struct {
  int64_t n_pages;                            /* 1 .. 2^31 - 1 */
  int32_t page;                               /* tokens in a page: 16, 32, 64, 128 or 256 */
  int32_t heads, dim;                         /* dim: a multiple of 16 up to CFP_CACHE_MAX_DIM */
  int32_t dtype;                              /* CFP_DT_F16, CFP_DT_BF16 or CFP_DT_E4M3 */
  void *k, *v;                                /* device, on 16 bytes */
  uint8_t *k_scale, *v_scale;                 /* device, on 16 bytes, for CFP_DT_E4M3; else NULL */
  int64_t k_page_stride, v_page_stride;       /* elements between pages, multiples of 16 */
  int64_t k_scale_page_stride, v_scale_page_stride;
} cfp_cache_desc;

/* Sequences of a call: rows starts[b] .. starts[b+1] - 1 of its tensors are the last tokens of sequence b, which has
 * lengths[b] tokens with them, so that row starts[b+1] - 1 is token lengths[b] - 1; token p lies in page
 * table[b][p / page] at p % page.  starts ascends within the call's rows; rows outside it are neither read nor written.
 * Several rows of the table may name one page to read it. */
typedef struct {
  int32_t n_seqs, width;   /* width: entries of a row of the table; width * page stays below 2^30 */
  const int32_t *table;    /* device [n_seqs][width], rows table_stride entries apart */
  int64_t table_stride;
  const int32_t *starts;   /* device [n_seqs + 1] */
  const int32_t *lengths;  /* device [n_seqs] */
  int32_t max_new;         /* the most rows that a sequence has, or more */
} cfp_sequences_desc;

/* Writes the keys and values of n_tokens rows (k, v [n_tokens][heads][dim] in CFP_DT_F16 or CFP_DT_BF16, strides in
 * elements, last dimension contiguous) to their places.  A cache of 16 bits is of the rows' type.  One of
 * CFP_DT_E4M3 gets for each token and head the least power of two 2^e, e >= -126, for which no finite entry passes
 * 448 2^e, and each entry over it rounded to the nearest value that is also one of the rows' type; infinities and NaN are
 * held as NaN.  A token whose place is before the first, behind the table's width or in a page outside the cache is not
 * written.  Where two rows have one place, what is held there afterwards is unspecified. */
int cfp_cache_write(const cfp_cache_desc *c, const cfp_sequences_desc *s, int64_t n_tokens, int32_t dtype, const void *k,
                    int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride,
                    int64_t v_head_stride, void *stream);

/* The tokens of the rows back, as the values that they stand for: k, v [n_tokens][heads][dim] contiguous, of the cache's type
 * or, from CFP_DT_E4M3, rounded to `dtype`: exact in the type that was written and in CFP_DT_BF16; in CFP_DT_F16 what was written
 * from CFP_DT_BF16 is an infinity beyond its range and has fewer bits below 2^-14.  A token before the first reads as zeros, one behind the table's width or in a page
 * outside the cache as NaN. */
int cfp_cache_read(const cfp_cache_desc *c, const cfp_sequences_desc *s, int64_t n_tokens, int32_t dtype, void *k, void *v,
                   void *stream);

/* ---- attention ---- */

typedef struct {
  int64_t n_tokens;
  int32_t n_q;            /* heads, a multiple of the cache's; head h reads the cache's head h / (n_q / heads) */
  int32_t dtype;          /* CFP_DT_F16 or CFP_DT_BF16: of q and out, and of a cache of 16 bits */
  const void *q;          /* device [n_tokens][n_q][dim], last dimension contiguous */
  int64_t q_token_stride, q_head_stride; /* in elements */
  float scale;            /* of the scores, > 0 */
  int32_t causal;         /* a row of token p sees the tokens up to p; else all of its sequence's */
  int32_t window;         /* and with window > 0 none before p - window + 1 */
} cfp_attend_desc;

/* out [n_tokens][n_q][dim]: for every row the mean of the values that it sees, weighted by exp(scale q . k); lse
 * [n_tokens][n_q] float (or NULL): the logarithm of the sum of the weights.  A row that sees nothing, or nothing but scores
 * of -infinity, gets zeros and -inf.  What a row does not see has no effect on it, whatever it holds: entries, and scales outside 1 to 254 too.
 * A value that a row sees and that is infinite, or no number, leaves the entry infinite or no number whatever its weight; which
 * of them is unspecified where the weight is zero.  Keys and values of CFP_DT_E4M3 are those that cfp_cache_read gives in `dtype`.  A row that sees a token of a page outside the
 * cache, and all rows of a sequence longer than its table or with more rows than max_new, become NaN.
 * The weights are rounded to `dtype` as operands of the product with the values; sums, maxima and what is held between
 * parts of a long sequence are in 32 bits.  The sums are divided at the end: bfloat16 values beyond 2^80 may leave the
 * range before, and of such below 2^-96 bits may be lost. */
size_t cfp_attend_workspace_bytes(const cfp_attend_desc *a, const cfp_cache_desc *c, const cfp_sequences_desc *s);
int cfp_attend(const cfp_attend_desc *a, const cfp_cache_desc *c, const cfp_sequences_desc *s, void *out, float *lse, void *ws,
               size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
