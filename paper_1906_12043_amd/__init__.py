"""MI355X-native hot path of CoCoD-SGD: one round of Algorithm 1 for W simulated workers on one GPU.

`binding` is a thin ctypes layer over libcocod.so (hand-written HIP for gfx950); it only marshals
arguments.  Build the library with `python -m paper_1906_12043_amd.build`.
"""
from .binding import (  # noqa: F401
    CocodError, Config, Context, lib, lib_path, plan_layout, debug_normals, debug_copy,
    cocod_create, cocod_destroy, cocod_local_steps, cocod_average_begin, cocod_average_end_apply,
    Grouped, CrossEntropy, grouped_workspace, grouped_forward, grouped_input_grad, grouped_weight_grad,
    cross_entropy_workspace, cross_entropy, checkpoint_store, checkpoint_load,
    debug_grouped_plan, debug_cross_entropy_plan,
    F32, BF16, F16, GROUPED_RELU_OUT, GROUPED_RELU_IN, GROUPED_FORWARD, GROUPED_INPUT_GRAD, GROUPED_WEIGHT_GRAD, CROSS_ENTROPY_SUM, CROSS_ENTROPY_RELU_IN,
    GRAD_QUADRATIC, GRAD_MLP, GRAD_EXTERNAL, SCHED_OVERLAP, SCHED_SERIAL, SCHED_FUSED, SCHED_HEAD, FLAG_DRY_RUN,
    OK, ERR_INVALID, ERR_STATE, ERR_HIP, ERR_NOMEM, ERR_UNSUPPORTED,
)
