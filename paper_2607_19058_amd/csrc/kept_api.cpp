// kept_api.cpp -- the C ABI declared in include/skew_kept.h: argument checks, then the launchers.
#include <hip/hip_runtime_api.h>

#include "moe_checks.h"
#include "moe_internal.h"
#include "kept_internal.h"

using namespace moe;

namespace {

int64_t lines(int64_t cols) { return (cols + 63) / 64 * 64; }   // a row stride in whole 128-byte lines
int64_t blocks_of(int64_t cols) { return (cols + SKEW_KEPT_BLOCK - 1) / SKEW_KEPT_BLOCK; }
// A work-group of 256 threads takes 128 blocks, and a launch has fewer than 2^32 threads.
constexpr int64_t kMostBlocks = ((int64_t)1 << 31) - 128;
bool kept_ok(int64_t rows, int64_t cols) {
  return rows >= 0 && cols_ok(cols) && rows <= kMostBlocks / blocks_of(cols);
}
constexpr int64_t kTileRows = 256;   // rows that a lane's 32-bit offset spans
bool codes_ok(const int8_t *codes, const uint8_t *scales) {
  return codes != nullptr && scales != nullptr && ((uintptr_t)codes & 15) == 0;
}
bool act_ok(const skew_act_desc *d) {
  if (d == nullptr || !kept_ok(d->rows, d->cols) || !type_ok(d->in_dtype) || !type_ok(d->out_dtype)) return false;
  if (d->kind < SKEW_ACT_RELU || d->kind > SKEW_ACT_GELU_TANH) return false;
  if ((d->codes_g == nullptr) != (d->scales_g == nullptr) || (d->codes_u == nullptr) != (d->scales_u == nullptr)) return false;
  return ((uintptr_t)d->codes_g & 15) == 0 && ((uintptr_t)d->codes_u & 15) == 0;
}
bool grad_kept_ok(const skew_rows *r, const skew_product_desc *p) {
  if (p == nullptr || p->x != nullptr || !type_ok(p->out_dtype) || !cols_ok(p->n)) return false;
  skew_product_desc q = *p;
  q.ldx = 32 * blocks_of(p->n);
  if (!product_ok(r, &q, true)) return false;
  const int64_t places = r->tokens * r->k;
  return kept_ok(places, p->n) && (p->out_dtype == SKEW_BF16 || places <= kMaxPlaces / 2);
}
// The workspace: restored rows (bf16 d: one a place; float32: those that are kept, as the product of a float32 d looks them up), then what
// the product needs, or rows of d where theirs do not begin at 16-byte positions.
struct KeptPlan {
  int64_t rows, ldx, ldd;   // ldd 0: d as it is
  size_t rest, bytes;
};
KeptPlan kept_plan(const skew_rows *r, const skew_product_desc *p) {
  const int64_t places = r->tokens * r->k, kept = p->flags & SKEW_GATHER ? r->tokens : places;
  KeptPlan k = {p->out_dtype == SKEW_F32 ? kept : places, lines(p->n), 0, 0, 0};
  k.rest = pad256((size_t)k.rows * k.ldx * 2);
  if (p->out_dtype == SKEW_F32) {
    skew_product_desc q = *p;
    q.ldx = k.ldx;
    k.bytes = k.rest + product_grad_f32_scratch(*r, q);
  } else {
    const bool as_is = ((uintptr_t)p->y & 15) == 0 && p->ldy % 8 == 0 && p->m % 8 == 0 && short_rows(kTileRows, p->ldy);
    if (!as_is) k.ldd = lines(p->m);
    k.bytes = k.rest + (size_t)places * k.ldd * 2;
  }
  return k;
}

}  // namespace

extern "C" {

int skew_keep8(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes, uint8_t *scales,
               void *stream) {
  if (!type_ok(dtype) || !kept_ok(rows, cols) || !ld_ok(ldx, cols, rows)) return SKEW_EINVAL;
  if (rows == 0) return SKEW_OK;
  if (x == nullptr || !codes_ok(codes, scales)) return SKEW_EINVAL;
  return status(launch_keep8(x, dtype, rows, cols, ldx, codes, scales, stream));
}

int skew_restore8(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int32_t dtype,
                  int64_t ldx, void *stream) {
  if (!type_ok(dtype) || !kept_ok(rows, cols) || !ld_ok(ldx, cols, rows)) return SKEW_EINVAL;
  if (rows == 0) return SKEW_OK;
  if (x == nullptr || !codes_ok(codes, scales)) return SKEW_EINVAL;
  return status(launch_restore8(codes, scales, rows, cols, x, dtype, ldx, stream));
}

int skew_expert_act(const skew_act_desc *d, void *stream) {
  if (!act_ok(d) || !ld_ok(d->ldg, d->cols, d->rows) || !ld_ok(d->lda, d->cols, d->rows)) return SKEW_EINVAL;
  if (d->codes_u != nullptr && (d->codes_g == nullptr || d->u == nullptr)) return SKEW_EINVAL;
  if (d->u != nullptr && !ld_ok(d->ldu, d->cols, d->rows)) return SKEW_EINVAL;
  if (d->rows == 0) return SKEW_OK;
  if (d->g == nullptr || d->a == nullptr) return SKEW_EINVAL;
  return status(launch_act(*d, stream));
}

int skew_expert_act_backward(const skew_act_desc *d, void *stream) {
  if (!act_ok(d) || !ld_ok(d->ldda, d->cols, d->rows) || !ld_ok(d->lddg, d->cols, d->rows)) return SKEW_EINVAL;
  if (d->a != nullptr && !ld_ok(d->lda, d->cols, d->rows)) return SKEW_EINVAL;
  if (d->codes_u != nullptr && !ld_ok(d->lddu, d->cols, d->rows)) return SKEW_EINVAL;
  if (d->rows == 0) return SKEW_OK;
  if (d->da == nullptr || d->dg == nullptr || d->codes_g == nullptr) return SKEW_EINVAL;
  if ((d->codes_u == nullptr) != (d->du == nullptr)) return SKEW_EINVAL;
  return status(launch_act_backward(*d, stream));
}

int skew_expert_matmul_grad_kept_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes) {
  if (!grad_kept_ok(r, p) || bytes == nullptr) return SKEW_EINVAL;
  *bytes = r->tokens > 0 ? kept_plan(r, p).bytes : 0;
  return SKEW_OK;
}

int skew_expert_matmul_grad_kept(const skew_rows *r, const skew_product_desc *p, const int8_t *codes, const uint8_t *scales,
                                 void *workspace, size_t workspace_bytes, void *stream) {
  if (!grad_kept_ok(r, p) || p->w == nullptr) return SKEW_EINVAL;
  if (r->tokens == 0) return status(launch_product_grad(*r, *p, stream));   // (nothing but dW is touched)
  if (p->y == nullptr || !codes_ok(codes, scales)) return SKEW_EINVAL;
  const KeptPlan k = kept_plan(r, p);
  if (workspace_bytes < k.bytes) return SKEW_ENOSPACE;
  if (workspace == nullptr) return SKEW_EINVAL;
  const bool gather = (p->flags & SKEW_GATHER) != 0;
  char *rest = static_cast<char *>(workspace) + k.rest;
  const int64_t whole = 32 * blocks_of(p->n);   // the columns past a row's end are 0, as their codes are
  int e = gather && p->out_dtype == SKEW_BF16
              ? launch_restore_places(*r, codes, scales, whole, workspace, k.ldx, stream)
              : launch_restore8(codes, scales, k.rows, whole, workspace, SKEW_BF16, k.ldx, stream);
  if (e != (int)hipSuccess) return SKEW_EHIP;
  if (p->out_dtype == SKEW_F32) {
    skew_product_desc q = *p;
    q.x = workspace;
    q.ldx = k.ldx;
    return status(launch_product_grad_f32(*r, q, rest, stream));
  }
  if (k.ldd > 0) e = launch_copy_rows(p->y, r->tokens * r->k, p->m, p->ldy, rest, k.ldd, stream);
  if (e != (int)hipSuccess) return SKEW_EHIP;
  return status(launch_grad_rows(*r, *p, workspace, k.ldx, k.ldd > 0 ? rest : p->y, k.ldd > 0 ? k.ldd : p->ldy, stream));
}

}  // extern "C"
