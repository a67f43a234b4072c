// head_api.cpp -- the C ABI declared in include/skew_loss.h: argument checks, then the launchers.
#include <hip/hip_runtime_api.h>

#include "head_internal.h"
#include "moe_checks.h"

using namespace moe;

namespace {

bool head_ok(const skew_head_desc *h) {
  if (h == nullptr || h->tokens < 0 || h->tokens > SKEW_MAX_LOSS_TOKENS || !cols_ok(h->vocab)) return false;
  if (h->d < 1 || h->d > SKEW_MAX_HEAD_WIDTH || (h->target_bytes != 4 && h->target_bytes != 8)) return false;
  if ((h->flags & ~SKEW_TRANSPOSE) != 0 || !(h->scale >= 1e-30f && h->scale <= 1e30f)) return false;
  const bool tied = (h->flags & SKEW_TRANSPOSE) != 0;
  return ld_ok(h->ldx, h->d, h->tokens) && ld_ok(h->ldw, tied ? h->d : h->vocab, tied ? h->vocab : h->d);
}
bool inputs_ok(const skew_head_desc *h) { return h->w != nullptr && (h->tokens == 0 || (h->x != nullptr && h->targets != nullptr)); }

}  // namespace

extern "C" {

int skew_head_loss_bytes(const skew_head_desc *h, size_t *bytes) {
  if (!head_ok(h) || bytes == nullptr) return SKEW_EINVAL;
  *bytes = h->tokens == 0 ? 0 : head_forward_scratch(*h);
  return SKEW_OK;
}

int skew_head_loss_backward_bytes(const skew_head_desc *h, size_t *bytes) {
  if (!head_ok(h) || bytes == nullptr) return SKEW_EINVAL;
  *bytes = h->tokens == 0 ? 0 : head_backward_scratch(*h);
  return SKEW_OK;
}

int skew_head_loss(const skew_head_desc *h, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  if (!head_ok(h) || !inputs_ok(h)) return SKEW_EINVAL;
  if (h->tokens == 0) return SKEW_OK;
  if (loss == nullptr || lse == nullptr) return SKEW_EINVAL;
  if (workspace_bytes < head_forward_scratch(*h)) return SKEW_ENOSPACE;
  if (workspace == nullptr) return SKEW_EINVAL;
  return status(launch_head_loss(*h, loss, lse, static_cast<char *>(workspace), stream));
}

int skew_head_loss_backward(const skew_head_desc *h, const float *lse, const float *dloss, const float *dlse, void *dx,
                            int32_t dx_dtype, int64_t lddx, void *dw, int64_t lddw, void *workspace,
                            size_t workspace_bytes, void *stream) {
  if (!head_ok(h) || !inputs_ok(h) || dw == nullptr || !type_ok(dx_dtype)) return SKEW_EINVAL;
  const bool tied = (h->flags & SKEW_TRANSPOSE) != 0;
  const int64_t rows = tied ? h->vocab : h->d, cols = tied ? h->d : h->vocab;
  if (!ld_ok(lddx, h->d, h->tokens) || !ld_ok(lddw, cols, rows)) return SKEW_EINVAL;
  if (h->tokens == 0) return status(launch_fill_zero(dw, rows, cols, lddw, stream));
  if (lse == nullptr || dloss == nullptr || dx == nullptr) return SKEW_EINVAL;
  if (workspace_bytes < head_backward_scratch(*h)) return SKEW_ENOSPACE;
  if (workspace == nullptr) return SKEW_EINVAL;
  return status(launch_head_loss_backward(*h, lse, dloss, dlse, dx, dx_dtype, lddx, dw, lddw, static_cast<char *>(workspace), stream));
}

}  // extern "C"
