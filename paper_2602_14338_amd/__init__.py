"""MI355X (gfx950) library for the per-token hot path of a group-based RL update.

The compute lives in hand-written HIP kernels behind a C ABI (include/aero.h, built into
libaero_hip.so next to this file).  This package is the thin Python binding: it marshals
torch tensors (device memory and streams only) into pointers and sizes.  There is no CPU
fallback: importing the binding without the built library raises.
"""
from .binding import (  # noqa: F401
    AdamWParams,
    AdvParams,
    AeroError,
    PreferenceParams,
    TensorTable,
    aero_adamw_moments,
    aero_adamw_step,
    aero_distill_loss_bwd,
    aero_embedding_bwd,
    aero_embedding_fwd,
    aero_grad_norm,
    aero_group_advantage,
    aero_grpo_loss_bwd,
    aero_grpo_loss_bwd_noalloc,
    aero_lmhead_logprob_fused,
    aero_logprob_fwd,
    aero_preference_loss,
    aero_preference_loss_bwd,
    aero_topk_logprob,
    aero_verify_draft,
    aero_workspace_bytes,
    library_path,
    AERO_F32,
    AERO_BF16,
    AERO_F16,
    AERO_F8E4M3,
    AERO_PAIR_HINGE,
    AERO_PAIR_LOGISTIC,
    AERO_PAIR_SQUARE,
    AERO_ROW_PADDING,
    AERO_ROW_UNTOUCHED,
    AERO_TAIL_BUCKET,
    AERO_TAIL_RENORM,
)
