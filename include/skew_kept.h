/*
 * skew_kept.h -- C ABI of what a training step keeps for its backward pass, in 8 bits, for AMD Instinct MI355X (gfx950).
 *
 * Rows are kept in 8 bits, the activation between an expert's products keeps its inputs in the pass that
 * computes it, and two backward passes read kept rows: the activation's, and the weights' gradient.
 *
 * Conventions are those of skew_moe.h (stream order, no allocation, no synchronisation, capture in a HIP graph, row strides in elements,
 * any alignment that an element type allows). Codes are 16-byte-aligned.
 */
#ifndef SKEW_KEPT_H
#define SKEW_KEPT_H

#include "skew_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of `cols` values (1 to SKEW_MAX_COLS) as dense codes int8 [rows x 32 B] and scales uint8 [rows x B], B = ceil(cols / 32):
 *   a block of 32 neighbours of a row has the scale s = 2^(b - 127), b its byte, 1 <= b <= 254. keep8 takes the smallest
 *   s >= 2^-126 with 127.5 s >= the block's largest finite magnitude, and 2^121 at most, so that values stay finite;
 *   code = x / s rounded to nearest even, -127 to 127; -128 where x is NaN or infinite;
 *   value = code s, NaN for -128. It is a bf16 number, off by s / 2 at most
 * (by s at most where |x| > 127.5 2^121). Codes past the end of a row are 0. bf16 rows: 1.03 of 2 bytes a value. */
#define SKEW_KEPT_BLOCK 32

/* Errors of each: SKEW_EINVAL, SKEW_EHIP. rows * ceil(cols / 32) <= 2^31 - 128; dtype SKEW_BF16 or SKEW_F32. */
int skew_keep8(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes, uint8_t *scales,
               void *stream);
int skew_restore8(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int32_t dtype,
                  int64_t ldx, void *stream);

enum { SKEW_ACT_RELU = 0, SKEW_ACT_SILU = 1, SKEW_ACT_GELU_TANH = 2 };

/* a = f(g) u, or f(g) where u is NULL; in float32, rounded once.
 *   relu       f(g) = max(g, 0), f'(0) = 0
 *   silu       f(g) = g s(g), s(y) = 1 / (1 + exp(-y))
 *   gelu_tanh  f(g) = g / 2 (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3)))
 * f(-inf) is its limit, 0; NaN gives NaN.
 * (Backward with relu, a g that is kept as 0, below half a step, takes no gradient.)
 * g, u: rows of cols in in_dtype. codes_g, scales_g, codes_u, scales_u: forward, where not NULL, get g and u as skew_keep8
 * makes them; backward, they are what is read (codes_u NULL: no u), g and u are not.
 * Backward, da (in_dtype) being a's gradient and g, u the kept values: a (NULL: not wanted) = f(g) u again, dg = da u f'(g),
 * du = da f(g). a, dg, du: out_dtype. */
typedef struct skew_act_desc {
  int64_t rows, cols;
  const void *g, *u, *da;
  void *a, *dg, *du;
  int64_t ldg, ldu, ldda, lda, lddg, lddu;
  int8_t *codes_g, *codes_u;
  uint8_t *scales_g, *scales_u;
  int32_t kind, in_dtype, out_dtype, reserved;
} skew_act_desc;

int skew_expert_act(const skew_act_desc *d, void *stream);
int skew_expert_act_backward(const skew_act_desc *d, void *stream);

/* skew_expert_matmul_grad() with the rows of x kept: tokens (SKEW_GATHER) or tokens * k rows of n values. p->x is NULL and
 * p->ldx not read; p->out_dtype is the type of d (p->y). The values are restored into the workspace, exactly, in bf16: a row for each place (tokens * k, also with
 * SKEW_GATHER), with a float32 d for each kept row. Rows of d at other than 16-byte positions are copied too. The size (host only)
 * depends on shapes and on d's alignment and stride.
 * Errors: SKEW_EINVAL, SKEW_ENOSPACE, SKEW_EHIP. */
int skew_expert_matmul_grad_kept_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes);
int skew_expert_matmul_grad_kept(const skew_rows *r, const skew_product_desc *p, const int8_t *codes, const uint8_t *scales,
                                 void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SKEW_KEPT_H */
