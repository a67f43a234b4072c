/*
 * skew_moe.h -- C ABI of the mixture-of-experts operators for AMD Instinct MI355X (gfx950).
 *
 * What a training step of a sparse model computes between its dense layers and the gradients
 * that skew_step() reads: the router's choice of experts, the experts' matrix products, the
 * token embedding, and the gradients of each (of the router's logits, of the stacked
 * (E, n, m) expert tensors and their inputs, of the embedding table).
 *
 * Conventions are those of skewadam.h: status codes, caller-owned device buffers, hipStream_t
 * as void*. Rows have 1 to SKEW_MAX_COLS columns. Every call is stream-ordered, launches nothing when it refuses its arguments,
 * allocates nothing, never synchronises, and can be captured in a HIP graph. Results are the
 * same bits on every run (no atomic adds of floats). Sums are float32; a result in bf16 is
 * rounded once. Row strides (ld*) are in elements. Pointers may have any alignment that their
 * element type allows; 16-byte-aligned rows are the fastest. Workspaces are 16-byte-aligned at
 * least. A call whose launch the device cannot take (some 2^24 work-groups: as many tokens, or tiles
 * of 64 x 128 results) returns SKEW_EHIP and leaves its outputs undefined.
 */
#ifndef SKEW_MOE_H
#define SKEW_MOE_H

#include "skewadam.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SKEW_BF16 = 0, SKEW_F32 = 1 };
enum { SKEW_SCORE_SOFTMAX = 0, SKEW_SCORE_SIGMOID = 1 };

#define SKEW_MAX_EXPERTS 1024
#define SKEW_MAX_CHOICES 16
#define SKEW_MAX_GROUPS 64
#define SKEW_MAX_COLS 16777216

/* How tokens choose experts. For a token's logits l_0 .. l_{E-1}:
 *   scores   s = softmax(l), or s_j = 1 / (1 + exp(-l_j)).
 *   values   v_j = l_j without a bias (the order of the scores), else s_j + bias_j. The bias takes
 *            part in the choice only, not in the weights.
 *   groups   the experts form `groups` runs of E / groups. With top_groups < groups only the
 *            top_groups groups of the highest value are open; a group's value is the sum of its
 *            group_sum (1 or 2) highest v.
 *   choice   the k open experts of the highest v, in that order. Ties go to the lowest index.
 *   weights  scale * s_i / (sum of s over the chosen) with renormalize, else scale * s_i.
 * A logit of -inf closes its expert: score 0, never chosen, and it adds nothing to its group's value (a
 * group without an open expert is never kept). A token with fewer than k open experts has expert -1
 * and weight 0 in the places left, down to a row of logits that are all -inf. NaN and +inf count
 * as the highest value, so they are chosen and show in the weights; with a bias, the other experts of
 * such a row have no softmax and follow by their bias alone. (With a bias, the sigmoid of +inf is a score of 1 like others.)
 *   tokens >= 0; 1 <= experts <= SKEW_MAX_EXPERTS; groups <= SKEW_MAX_GROUPS divides experts;
 *   1 <= top_groups <= groups; 1 <= k <= SKEW_MAX_CHOICES, k <= top_groups * experts / groups;
 *   group_sum 2 needs a bias (sums of logits are no score);
 *   dtype of the logits (SKEW_BF16, SKEW_F32), ld >= experts their row stride; scale finite. */
typedef struct skew_route_desc {
  int64_t tokens, ld;
  int32_t experts, k, dtype, score;
  int32_t groups, top_groups, group_sum, renormalize;
  float scale;
  int32_t reserved;
} skew_route_desc;

/* logits device [tokens x ld]; bias device float [experts] or NULL; weights float and chosen int32
 * [tokens x k]. Errors: SKEW_EINVAL, SKEW_EHIP. */
int skew_route(const skew_route_desc *d, const void *logits, const float *bias, float *weights, int32_t *chosen,
               void *stream);

/* The gradient of the logits, dense [tokens x experts] in the logits' type, from that of the
 * weights (float [tokens x k]) and the choice that skew_route made (entries outside [0, experts)
 * are none). The choice itself has no gradient, nor has the bias, so the fields of the choice
 * (groups, top_groups, group_sum) are not read. Errors: SKEW_EINVAL, SKEW_EHIP. */
int skew_route_backward(const skew_route_desc *d, const void *logits, const int32_t *chosen, const float *dweights,
                        void *dlogits, void *stream);

/* Scratch bytes of skew_expert_rows() for n choices and of skew_embed_grad() for n tokens of a
 * `keys` x `cols` table (cols 0: skew_expert_rows). Host only. Errors: SKEW_EINVAL. */
int skew_order_bytes(int64_t n, int64_t keys, int64_t cols, size_t *bytes);

/* The (token, choice) pairs in the order of their experts, and of their index within an expert:
 *   chosen   int32 [n], n = tokens * k < 2^31; entries outside [0, experts) are none.
 *   offsets  OUT int32 [experts + 1]: expert e holds places offsets[e] .. offsets[e + 1).
 *   rows     OUT int32 [n]: the pair at each place; -1 from place offsets[experts] on.
 *   slots    OUT int32 [n]: the place of each pair, -1 where it has no expert.
 * Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_expert_rows(const int32_t *chosen, int64_t n, int32_t experts, int32_t *offsets, int32_t *rows,
                     int32_t *slots, void *workspace, size_t workspace_bytes, void *stream);

/* The order that skew_expert_rows made, as the products take it. */
typedef struct skew_rows {
  const int32_t *offsets, *rows, *slots;
  int64_t tokens;
  int32_t k, experts;
} skew_rows;

enum { SKEW_GATHER = 1, SKEW_TRANSPOSE = 2 };

/* y[p] = s_p a_p W[e] for every place p of every expert e (SKEW_TRANSPOSE: s_p a_p W[e]^T).
 *   x      bf16: a_p is row p of x (tokens * k rows), or with SKEW_GATHER the row of p's token
 *          (tokens rows).
 *   w      bf16 (experts, n, m), row stride ldw >= m, slice stride slice >= n * ldw.
 *   scale  NULL (s_p = 1), or float [tokens x k]: s_p is the entry of p's pair.
 *   y      tokens * k rows in out_dtype; rows past the last expert's are set to zero.
 *   n, m >= 1. ldx >= n and ldy >= m (swapped with SKEW_TRANSPOSE).
 * skew_expert_matmul_bytes() gives the scratch (host only; it depends on shapes alone).
 * Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
typedef struct skew_product_desc {
  const void *x;
  const void *w;
  void *y;
  const float *scale;
  int64_t n, m, ldx, ldw, slice, ldy;
  int32_t flags, out_dtype;
} skew_product_desc;

int skew_expert_matmul_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes);
int skew_expert_matmul(const skew_rows *r, const skew_product_desc *p, void *workspace, size_t workspace_bytes,
                       void *stream);

/* dW[e] = sum over e's places of a_p^T d_p, bf16 (experts, n, m) with strides ldw, slice: the
 * weights' gradient, zero for experts without rows. x, scale and flags (SKEW_GATHER) as above with
 * scale NULL; y holds d (bf16, tokens * k rows of m, stride ldy) and is only read; w is written.
 * Errors: SKEW_EINVAL, SKEW_EHIP. */
int skew_expert_matmul_grad(const skew_rows *r, const skew_product_desc *p, void *stream);

/* The same with d in float32 (ldy in floats). The matrix cores take it as the sum of two bf16 numbers,
 * which leaves out at most 2^-16 of a value; the contraction is twice as long, so it takes up to twice the time.
 * tokens * k < 2^30. skew_expert_matmul_grad_f32_bytes() gives the scratch (host only; it depends on
 * shapes alone). Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_expert_matmul_grad_f32_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes);
int skew_expert_matmul_grad_f32(const skew_rows *r, const skew_product_desc *p, void *workspace,
                                size_t workspace_bytes, void *stream);

/* out[t] = sum over t's choices j of weights[t, j] y[place of (t, j)] (weights NULL: 1). A token without
 * experts gets zeros. y: tokens * k rows of m in y_dtype; out: tokens rows in out_dtype.
 * Errors: SKEW_EINVAL, SKEW_EHIP. */
int skew_expert_combine(const skew_rows *r, const void *y, int32_t y_dtype, int64_t ldy, const float *weights,
                        void *out, int32_t out_dtype, int64_t ldo, int64_t m, void *stream);

/* Its gradients: dy[p] = weights[t, j] dout[t] (bf16, rows past the last expert's zero) and
 * dweights[t, j] = <dout[t], y[p]> (float [tokens x k], 0 where the pair has no expert). dout bf16.
 * Errors: SKEW_EINVAL, SKEW_EHIP. */
int skew_expert_combine_backward(const skew_rows *r, const void *dout, int64_t ldo, const void *y, int32_t y_dtype,
                                 int64_t ldy, const float *weights, void *dy, int64_t lddy, float *dweights,
                                 int64_t m, void *stream);

/* The same with dy in float32, for a gradient of the weights that is rounded once:
 * skew_expert_matmul_grad_f32() takes these rows as they are. */
int skew_expert_combine_backward_f32(const skew_rows *r, const void *dout, int64_t ldo, const void *y, int32_t y_dtype,
                                     int64_t ldy, const float *weights, float *dy, int64_t lddy, float *dweights,
                                     int64_t m, void *stream);

/* Rows of an embedding table. ids: int32 or int64 (id_bytes 4 or 8) [tokens]; an id outside
 * [0, vocab) is no token: its row of `out` is zero and it adds nothing to the gradient.
 *   skew_embed       out[t] = scale * table[id_t]
 *   skew_embed_grad  dtable[v] = scale * sum of dout[t] over the t with id_t = v, every row of it
 *                    written (zero where no token has the id); a row's tokens are added in
 *                    order, in runs that end at multiples of 32 places of all
 *                    tokens sorted by id, and then the runs.
 * table, out, dout and dtable share `dtype`; rows of `cols` at strides ld*. tokens < 2^31,
 * vocab < 2^31. Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_embed(const void *ids, int32_t id_bytes, int64_t tokens, const void *table, int64_t vocab, int64_t cols,
               int64_t ldt, void *out, int64_t ldo, int32_t dtype, float scale, void *stream);
int skew_embed_grad(const void *ids, int32_t id_bytes, int64_t tokens, const void *dout, int64_t ldo, void *dtable,
                    int64_t vocab, int64_t cols, int64_t ldt, int32_t dtype, float scale, void *workspace,
                    size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SKEW_MOE_H */
