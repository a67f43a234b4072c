// kept_internal.h -- launchers of the rows kept in 8 bits.
#pragma once

#include <type_traits>

#include "../../include/skew_kept.h"

namespace moe {

int launch_keep8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes, uint8_t *scales, void *stream);
int launch_restore8(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int dtype, int64_t ldx,
                    void *stream);
int launch_act(const skew_act_desc &d, void *stream);
int launch_act_backward(const skew_act_desc &d, void *stream);

}  // namespace moe
