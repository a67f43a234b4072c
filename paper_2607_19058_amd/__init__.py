"""SkewAdam optimizer step for AMD Instinct MI355X (gfx950): HIP kernels behind a C ABI."""
from .skewadam import (BACKBONE, EXPERT, ROUTER, TIERS, STATE_MOMENTUM, STATE_FACTORED, STATE_FP32,  # noqa: F401
                       FLAG_EXACT_CLIP, FLAG_EXACT_ULP, SkewAdam, SkewError, HParams, TensorDesc, lib, make_desc,
                       state_bytes)
from .moe import (ExpertRows, embed, embed_grad, expert_combine, expert_combine_backward, expert_matmul,  # noqa: F401
                  expert_matmul_grad, expert_rows, route, route_backward)
