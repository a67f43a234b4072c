// moe_api.cpp -- the C ABI declared in include/skew_moe.h: argument checks, then the launchers.
#include <hip/hip_runtime_api.h>

#include <cmath>

#include "moe_checks.h"
#include "moe_internal.h"

using namespace moe;

namespace {

bool route_ok(const skew_route_desc *d) {
  if (d == nullptr || d->tokens < 0 || !type_ok(d->dtype)) return false;
  if (d->score != SKEW_SCORE_SOFTMAX && d->score != SKEW_SCORE_SIGMOID) return false;
  if (d->experts < 1 || d->experts > SKEW_MAX_EXPERTS || !ld_ok(d->ld, d->experts, d->tokens)) return false;
  if (d->k < 1 || d->k > SKEW_MAX_CHOICES || d->k > d->experts) return false;
  if (d->renormalize != 0 && d->renormalize != 1) return false;
  return d->tokens <= kMaxPlaces / d->k && std::isfinite(d->scale);
}
bool groups_ok(const skew_route_desc *d, const float *bias) {
  if (d->groups < 1 || d->groups > SKEW_MAX_GROUPS || d->experts % d->groups != 0) return false;
  if (d->top_groups < 1 || d->top_groups > d->groups) return false;
  if (d->k > (int64_t)d->top_groups * (d->experts / d->groups)) return false;
  return d->group_sum == 1 || (d->group_sum == 2 && bias != nullptr);
}

}  // namespace

extern "C" {

int skew_route(const skew_route_desc *d, const void *logits, const float *bias, float *weights, int32_t *chosen,
               void *stream) {
  if (!route_ok(d) || !groups_ok(d, bias)) return SKEW_EINVAL;
  if (d->tokens == 0) return SKEW_OK;
  if (logits == nullptr || weights == nullptr || chosen == nullptr) return SKEW_EINVAL;
  return status(launch_route(*d, logits, bias, weights, chosen, stream));
}

int skew_route_backward(const skew_route_desc *d, const void *logits, const int32_t *chosen, const float *dweights,
                        void *dlogits, void *stream) {
  if (!route_ok(d)) return SKEW_EINVAL;
  if (d->tokens == 0) return SKEW_OK;
  if (logits == nullptr || chosen == nullptr || dweights == nullptr || dlogits == nullptr) return SKEW_EINVAL;
  return status(launch_route_backward(*d, logits, chosen, dweights, dlogits, stream));
}

int skew_order_bytes(int64_t n, int64_t keys, int64_t cols, size_t *bytes) {
  if (n < 0 || n > kMaxPlaces || keys < 1 || keys > kMaxPlaces || cols < 0 || cols > kMaxCols) return SKEW_EINVAL;
  if (bytes == nullptr) return SKEW_EINVAL;
  *bytes = sort_plan(n, keys).bytes + (cols > 0 ? embed_scratch(n, cols) : 0);
  return SKEW_OK;
}

int skew_expert_rows(const int32_t *chosen, int64_t n, int32_t experts, int32_t *offsets, int32_t *rows,
                     int32_t *slots, void *workspace, size_t workspace_bytes, void *stream) {
  if (n < 0 || n > kMaxPlaces || experts < 1 || experts > SKEW_MAX_EXPERTS || offsets == nullptr) return SKEW_EINVAL;
  if (n > 0 && (chosen == nullptr || rows == nullptr || slots == nullptr)) return SKEW_EINVAL;
  const SortPlan p = sort_plan(n, experts);
  if (workspace_bytes < p.bytes) return SKEW_ENOSPACE;
  if (p.bytes > 0 && workspace == nullptr) return SKEW_EINVAL;
  SortOut o;
  o.offsets = offsets;
  o.rows = rows;
  o.slots = slots;
  return status(launch_sort(p, chosen, 4, static_cast<char *>(workspace), &o, stream));
}

int skew_expert_matmul_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes) {
  if (!product_ok(r, p, false) || bytes == nullptr) return SKEW_EINVAL;
  *bytes = product_scratch(*r, *p);
  return SKEW_OK;
}

int skew_expert_matmul(const skew_rows *r, const skew_product_desc *p, void *workspace, size_t workspace_bytes,
                       void *stream) {
  if (!product_ok(r, p, false)) return SKEW_EINVAL;
  if (r->tokens == 0) return SKEW_OK;
  if (p->x == nullptr || p->w == nullptr || p->y == nullptr) return SKEW_EINVAL;
  const size_t need = product_scratch(*r, *p);
  if (workspace_bytes < need) return SKEW_ENOSPACE;
  if (need > 0 && workspace == nullptr) return SKEW_EINVAL;
  return status(launch_product(*r, *p, static_cast<char *>(workspace), stream));
}

int skew_expert_matmul_grad(const skew_rows *r, const skew_product_desc *p, void *stream) {
  if (!product_ok(r, p, true) || p->w == nullptr) return SKEW_EINVAL;
  if (r->tokens > 0 && (p->x == nullptr || p->y == nullptr)) return SKEW_EINVAL;
  return status(launch_product_grad(*r, *p, stream));
}

int skew_expert_matmul_grad_f32_bytes(const skew_rows *r, const skew_product_desc *p, size_t *bytes) {
  if (!product_ok(r, p, true) || r->tokens * r->k > kMaxPlaces / 2 || bytes == nullptr) return SKEW_EINVAL;
  *bytes = product_grad_f32_scratch(*r, *p);
  return SKEW_OK;
}

int skew_expert_matmul_grad_f32(const skew_rows *r, const skew_product_desc *p, void *workspace,
                                size_t workspace_bytes, void *stream) {
  if (!product_ok(r, p, true) || r->tokens * r->k > kMaxPlaces / 2 || p->w == nullptr) return SKEW_EINVAL;
  if (r->tokens == 0) return status(launch_product_grad(*r, *p, stream));   // (d is not read)
  if (p->x == nullptr || p->y == nullptr) return SKEW_EINVAL;
  if (workspace_bytes < product_grad_f32_scratch(*r, *p)) return SKEW_ENOSPACE;
  if (workspace == nullptr) return SKEW_EINVAL;
  return status(launch_product_grad_f32(*r, *p, static_cast<char *>(workspace), stream));
}

int skew_expert_combine(const skew_rows *r, const void *y, int32_t y_dtype, int64_t ldy, const float *weights,
                        void *out, int32_t out_dtype, int64_t ldo, int64_t m, void *stream) {
  if (!rows_ok(r) || !type_ok(y_dtype) || !type_ok(out_dtype) || !cols_ok(m)) return SKEW_EINVAL;
  if (!ld_ok(ldy, m, r->tokens * r->k) || !ld_ok(ldo, m, r->tokens)) return SKEW_EINVAL;
  if (r->tokens == 0) return SKEW_OK;
  if (y == nullptr || out == nullptr) return SKEW_EINVAL;
  return status(launch_combine(*r, y, y_dtype, ldy, weights, out, out_dtype, ldo, m, stream));
}

namespace {
int combine_backward(const skew_rows *r, const void *dout, int64_t ldo, const void *y, int32_t y_dtype, int64_t ldy,
                     const float *weights, void *dy, int dy_dtype, int64_t lddy, float *dweights, int64_t m,
                     void *stream) {
  if (!rows_ok(r) || !type_ok(y_dtype) || !cols_ok(m)) return SKEW_EINVAL;
  const int64_t places = r->tokens * r->k;
  if (!ld_ok(ldo, m, r->tokens) || !ld_ok(ldy, m, places) || !ld_ok(lddy, m, places)) return SKEW_EINVAL;
  if (r->tokens == 0) return SKEW_OK;
  if (dout == nullptr || y == nullptr || dy == nullptr || dweights == nullptr) return SKEW_EINVAL;
  return status(launch_combine_backward(*r, dout, ldo, y, y_dtype, ldy, weights, dy, dy_dtype, lddy, dweights, m, stream));
}
}  // namespace

int skew_expert_combine_backward(const skew_rows *r, const void *dout, int64_t ldo, const void *y, int32_t y_dtype,
                                 int64_t ldy, const float *weights, void *dy, int64_t lddy, float *dweights,
                                 int64_t m, void *stream) {
  return combine_backward(r, dout, ldo, y, y_dtype, ldy, weights, dy, SKEW_BF16, lddy, dweights, m, stream);
}

int skew_expert_combine_backward_f32(const skew_rows *r, const void *dout, int64_t ldo, const void *y, int32_t y_dtype,
                                     int64_t ldy, const float *weights, float *dy, int64_t lddy, float *dweights,
                                     int64_t m, void *stream) {
  return combine_backward(r, dout, ldo, y, y_dtype, ldy, weights, dy, SKEW_F32, lddy, dweights, m, stream);
}

int skew_embed(const void *ids, int32_t id_bytes, int64_t tokens, const void *table, int64_t vocab, int64_t cols,
               int64_t ldt, void *out, int64_t ldo, int32_t dtype, float scale, void *stream) {
  if ((id_bytes != 4 && id_bytes != 8) || tokens < 0 || tokens > kMaxPlaces || vocab < 1 || vocab > kMaxPlaces)
    return SKEW_EINVAL;
  if (!type_ok(dtype) || !cols_ok(cols) || !ld_ok(ldt, cols, vocab) || !ld_ok(ldo, cols, tokens)) return SKEW_EINVAL;
  if (!std::isfinite(scale)) return SKEW_EINVAL;
  if (tokens == 0) return SKEW_OK;
  if (ids == nullptr || table == nullptr || out == nullptr) return SKEW_EINVAL;
  return status(launch_embed(ids, id_bytes, tokens, table, vocab, cols, ldt, out, ldo, dtype, scale, stream));
}

int skew_embed_grad(const void *ids, int32_t id_bytes, int64_t tokens, const void *dout, int64_t ldo, void *dtable,
                    int64_t vocab, int64_t cols, int64_t ldt, int32_t dtype, float scale, void *workspace,
                    size_t workspace_bytes, void *stream) {
  if ((id_bytes != 4 && id_bytes != 8) || tokens < 0 || tokens > kMaxPlaces || vocab < 1 || vocab > kMaxPlaces)
    return SKEW_EINVAL;
  if (!type_ok(dtype) || !cols_ok(cols) || !ld_ok(ldt, cols, vocab) || !ld_ok(ldo, cols, tokens)) return SKEW_EINVAL;
  if (!std::isfinite(scale) || dtable == nullptr) return SKEW_EINVAL;
  if (tokens > 0 && (ids == nullptr || dout == nullptr)) return SKEW_EINVAL;
  const SortPlan p = sort_plan(tokens, vocab);
  if (workspace_bytes < p.bytes + embed_scratch(tokens, cols)) return SKEW_ENOSPACE;
  if (p.bytes > 0 && workspace == nullptr) return SKEW_EINVAL;
  char *ws = static_cast<char *>(workspace);
  SortOut o;
  if (tokens > 0) {
    const int e = launch_sort(p, ids, id_bytes, ws, &o, stream);
    if (e != (int)hipSuccess) return SKEW_EHIP;
  }
  return status(launch_embed_grad(o, tokens, dout, ldo, dtable, vocab, cols, ldt, dtype, scale, ws + p.bytes, stream));
}

}  // extern "C"
