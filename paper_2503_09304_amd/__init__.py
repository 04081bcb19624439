"""qmoe: a priority-ordered, preemptible Mixture-of-Experts layer for AMD MI355X (gfx950).

The work is done by libqmoe.so (hand-written HIP kernels behind the C ABI of include/qmoe.h, and
the host scheduler of include/qsched.h).
This package only marshals arguments; there is no CPU or PyTorch fallback, and loading fails
loudly when the library has not been built (python -m paper_2503_09304_amd.build)."""
from .binding import (  # noqa: F401
    MOE_BF16,
    MOE_CLASS_ALL,
    MOE_Y_F32,
    MOE_CLASS_BE,
    MOE_CLASS_LS,
    MOE_DONE,
    MOE_E_ARG,
    MOE_E_HIP,
    MOE_E_INCOMPLETE,
    MOE_E_STATE,
    MOE_E_WORKSPACE,
    MOE_F32,
    MOE_OK,
    MOE_W_MXFP4,
    MOE_W_MXFP4_ROWMAJOR,
    MOE_W_PACKED,
    MOE_W_ROWMAJOR,
    SCHED_BE,
    SCHED_DECODE,
    SCHED_E_ARG,
    SCHED_E_JOB,
    SCHED_LS,
    SCHED_NONE,
    SCHED_OK,
    SCHED_PREFILL,
    SCHED_Q_BE_DECODE,
    SCHED_Q_BE_PREFILL,
    SCHED_Q_LS_DECODE,
    SCHED_Q_LS_PREFILL,
    UINT32_MAX,
    Context,
    MoeConfig,
    MoeCursor,
    MoeError,
    MoeUnit,
    MoeWeights,
    SchedBatch,
    SchedError,
    Scheduler,
    lib,
    lib_path,
    moe_last_error,
    moe_pack_weights,
    moe_probe_mfma,
    moe_route_noalloc,
    moe_plan_units,
    moe_workspace_bytes,
)

# The attention calls (include/qattn.h) work on torch tensors; their module, and torch with it, is imported at first use.
_ATTENTION = ("ATTN_BF16", "ATTN_FP8", "AttnCache", "AttnRope", "attn_append", "attn_decode", "attn_decode_workspace", "attn_prompt", "attn_read",
              "attn_rope_frequencies")


def __getattr__(name):
    if name not in _ATTENTION:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from . import attention
    value = globals()[name] = getattr(attention, name)
    return value
