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
// Which tile: us with tiles of 256 x 256, 128 x 256 and 64 x 128, and from rows in bf16 (moe_product.hip, which looks them up):
//   32 experts of 2048 x 8192, uneven rows, mean   32   314 227 292 | 275          8 experts of 1024 x 1024, 1024 rows   42  37  35 | 32
//                                                 128   388 343 420 | 394          8 of 256 x 1024, 250                  21  21  21 | 15
//                                                 256   483 486 565 | 505          8 of 2048 x 2048, 2048               126 144 192 | 122
//                                                 512   677 713 880 | 710          4 of 2048 x 8192, 2048               223 250 331 | 237
//   16 experts of 2765 x 1031, 563 rows                 108  99 116 | 115          128 of 512 x 2048, 128               105 103 131 | 110
inline int kept_tile(int64_t places, int64_t experts, int64_t n, int64_t m) {   // 0, 1, 2 of these
  const int64_t rows = places / experts;   // of an expert, on average
  auto tiles = [&](int64_t bm, int64_t bn) { return experts * ((n + bm - 1) / bm) * ((m + bn - 1) / bn); };
  if ((rows >= 384 && tiles(256, 256) >= 2048) || (rows >= 1024 && tiles(256, 256) >= 512)) return 0;
  return tiles(128, 256) >= 512 ? 1 : 2;
}
int launch_act(const skew_act_desc &d, void *stream);
int launch_act_backward(const skew_act_desc &d, void *stream);

}  // namespace moe
