// moe_checks.h -- argument checks that the C ABIs of the operators share.
#pragma once

#include <hip/hip_runtime_api.h>

#include "../../include/skew_moe.h"

namespace moe {

constexpr int64_t kMaxPlaces = 0x7FFFFFFF;   // pairs and ids have 32-bit indices
constexpr int64_t kMaxCols = 1 << 24;        // columns of a row
constexpr int64_t kMaxSpan = (int64_t)1 << 59;   // elements that a strided tensor may span

inline int status(int hip_error) { return hip_error == (int)hipSuccess ? SKEW_OK : SKEW_EHIP; }

inline bool type_ok(int32_t t) { return t == SKEW_BF16 || t == SKEW_F32; }
inline bool cols_ok(int64_t c) { return c >= 1 && c <= kMaxCols; }
// a stride that holds its row and does not overflow over the rows
inline bool ld_ok(int64_t ld, int64_t cols, int64_t rows) {
  return ld >= cols && (rows <= 1 || ld <= kMaxSpan / rows);
}

inline bool rows_ok(const skew_rows *r) {
  if (r == nullptr || r->tokens < 0 || r->k < 1 || r->k > SKEW_MAX_CHOICES) return false;
  if (r->experts < 1 || r->experts > SKEW_MAX_EXPERTS || r->tokens > kMaxPlaces / r->k) return false;
  return r->offsets != nullptr && (r->tokens == 0 || (r->rows != nullptr && r->slots != nullptr));
}
inline bool product_ok(const skew_rows *r, const skew_product_desc *p, bool grad) {
  if (!rows_ok(r) || p == nullptr || !cols_ok(p->n) || !cols_ok(p->m)) return false;
  if ((p->flags & ~(grad ? SKEW_GATHER : SKEW_GATHER | SKEW_TRANSPOSE)) != 0) return false;
  if (grad ? p->scale != nullptr : !type_ok(p->out_dtype)) return false;
  const bool back = (p->flags & SKEW_TRANSPOSE) != 0;
  const int64_t places = r->tokens * r->k, in = back ? p->m : p->n, out = back ? p->n : p->m;
  if (!ld_ok(p->ldx, in, p->flags & SKEW_GATHER ? r->tokens : places) || !ld_ok(p->ldy, out, places)) return false;
  if (!ld_ok(p->ldw, p->m, p->n) || p->slice < p->n * p->ldw || !ld_ok(p->slice, 1, r->experts)) return false;
  return true;
}

}  // namespace moe
