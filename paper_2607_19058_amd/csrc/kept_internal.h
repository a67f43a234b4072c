// kept_internal.h -- launchers of the rows kept in 8 bits.
#pragma once

#include <type_traits>

#include "../../include/skew_kept.h"

namespace moe {

int launch_keep8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes, uint8_t *scales, void *stream);
int launch_restore8(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int dtype, int64_t ldx,
                    void *stream);
// x of each place p: the kept row rows[p] / k (places without a pair: not written)
int launch_restore_places(const skew_rows &r, const int8_t *codes, const uint8_t *scales, int64_t cols, void *x, int64_t ldx, void *stream);
int launch_copy_rows(const void *x, int64_t rows, int64_t cols, int64_t ldx, void *y, int64_t ldy, void *stream);   // bf16, zeros up to ldy
// skew_expert_matmul_grad of rows of x and d, one a place, at 16-byte positions (their columns padded to multiples of 8)
int launch_grad_rows(const skew_rows &r, const skew_product_desc &p, const void *x, int64_t ldx, const void *d, int64_t ldd, void *stream);
int launch_act(const skew_act_desc &d, void *stream);
int launch_act_backward(const skew_act_desc &d, void *stream);

}  // namespace moe
