/*
 * skew_loss.h -- C ABI of the head's loss for AMD Instinct MI355X (gfx950): softmax cross entropy over a vocabulary from
 * the rows before the head and the head's weights, and the gradients of both, without ever holding the logits.
 *
 * Conventions are those of skew_moe.h (stream order, no allocation, no synchronisation, capture in a HIP graph, the same bits on
 * every run, row strides in elements, any alignment that an element type allows).
 */
#ifndef SKEW_LOSS_H
#define SKEW_LOSS_H

#include "skew_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SKEW_MAX_LOSS_TOKENS 4194304
#define SKEW_MAX_HEAD_WIDTH 1048576

/* For token t with row x_t and target y_t, over the words v of the vocabulary:
 *   z_tv   = scale <x_t, w_v>             (float32 sums of bf16 products)
 *   lse_t  = log sum_v exp(z_tv)
 *   loss_t = lse_t - z_t,y_t
 * A target outside [0, vocab) is no token: loss and lse are 0, its row of x is not looked at (it may hold NaN), its row of dx is zero,
 * and it adds nothing to dw.
 * Gradients, from those of loss (dloss) and lse (dlse; NULL: 0), G being that of the logits:
 *   G_tv = scale ((dloss_t + dlse_t) exp(z_tv - lse_t) - dloss_t [v = y_t]);   dx = G w^T;   dw = x^T G
 * computed in pieces of the vocabulary. G is rounded before these products: up to 512 tokens, or 2^29 of
 * tokens * d * vocab, to the sum of two bf16 numbers, which leaves out 2^-16 of an entry; with more, G and the operand beside it are float16 numbers (11 bits, 8 times finer than bf16) times powers
 * of two: of G's rows, by their tokens' larger factor, and of the columns of x and w (their d), by their largest values. So an entry
 * of G below 2^-27 of its row's factor, or one of x or w below 2^-28 of its column's largest, can keep fewer bits, down to none 11 powers
 * further (for dw, of x times its token's factor). For dw a word of which every entry of G is below 2^-31 sqrt(tokens) of its row's factor is
 * computed again beside a power of two of its own (words between that and 2^-30 sqrt(tokens) may be), so that rare words keep 11 bits of
 * their largest entry; calls with many such words take longer. dx and dw are rounded once more.
 * NaN and infinities in x and w give NaN where they reach; a logit of +inf gives NaN.
 *   x      bf16 [tokens x d], row stride ldx;  0 <= tokens <= SKEW_MAX_LOSS_TOKENS;  1 <= d <= SKEW_MAX_HEAD_WIDTH
 *   w      bf16: column v of [d x vocab] is word v; with SKEW_TRANSPOSE row v of [vocab x d], as an embedding's
 *          table is; row stride ldw;  1 <= vocab <= SKEW_MAX_COLS
 *   targets int32 or int64 (target_bytes 4 or 8) [tokens]
 *   scale  from 1e-30 to 1e30 */
typedef struct skew_head_desc {
  const void *x, *w, *targets;
  int64_t tokens, d, vocab, ldx, ldw;
  int32_t target_bytes, flags;
  float scale;
  int32_t reserved;
} skew_head_desc;

/* Scratch bytes of the two calls (host only; they depend on shapes, strides and alignments). Errors: SKEW_EINVAL. Copies are made of x or w where
 * its rows do not begin at 16-byte positions or are more than 4178004 elements apart, or d (of an untied w, vocab too) is no multiple of 8.
 *   forward   8 bytes for each row and 64 or 128 words (1/16 or 1/32 of the logits in bf16), of 16384 tokens at most;
 *             the copies: x of these tokens, and 512 MiB of w at most
 *   backward  G of a piece of the vocabulary in 16 bits, or twice 16: 512 MiB, or 256 words where that is more (512 bytes a token, or
 *             1024), at most; where G is float16, the piece's words in float16; x in 16 bits, once or twice; the copies of x and of the piece's
 *             words; float32 dx where there are several pieces; float32 parts of dx and dw that several work-groups share.
 *             Rows in the workspace are up to 136 elements longer than their values, pieces up to 256 words longer.
 *             8192 tokens, 50304 words of width 2048: 647 MB (bf16 logits: 824); 4096 tokens: 704 (412), as all of G is one piece. */
int skew_head_loss_bytes(const skew_head_desc *h, size_t *bytes);
int skew_head_loss_backward_bytes(const skew_head_desc *h, size_t *bytes);

/* loss, lse: float [tokens]. Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_head_loss(const skew_head_desc *h, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* lse as skew_head_loss gave it. dx [tokens x d] in dx_dtype, stride lddx; dw bf16 in w's layout, stride lddw, every row of it
 * written. Outputs share no memory with inputs, which are read after parts of the outputs are written. Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_head_loss_backward(const skew_head_desc *h, const float *lse, const float *dloss, const float *dlse, void *dx,
                            int32_t dx_dtype, int64_t lddx, void *dw, int64_t lddw, void *workspace,
                            size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SKEW_LOSS_H */
