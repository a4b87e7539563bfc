"""Leapfrogging backpropagation for one MI355X: Python binding of liblf.so.

The binding marshals arguments only; every step of the pass runs in the HIP
kernels of the library.  PyTorch is used for device memory and streams.
"""
from .binding import (  # noqa: F401
    LF_OK, LF_EINVAL, LF_ESTATE, LF_ENOMEM, LF_EHIP, LF_EUNSUPPORTED,
    LF_F32, LF_BF16, LF_COST_QUADRATIC,
    LF_SCHED_AUTO, LF_SCHED_STREAMS, LF_SCHED_PERSISTENT, LF_SCHED_REDUNDANT, LF_SCHED_FUSED, LF_DEBUG_CHAIN_ONLY,
    LfError, lib, library_path,
    lf_workspace_bytes, lf_create, lf_workspace_bytes_widths, lf_create_widths,
    lf_set_params, lf_set_grad_buffers, lf_set_schedule, lf_set_debug_flags, lf_set_cost_scale, lf_set_sgd, lf_set_master_weights,
    lf_forward, lf_backward_leapfrog, lf_backward_leapfrog_noalloc, lf_noalloc_scratch_limit, lf_grads, lf_activations, lf_schedule_worker, lf_algorithm1_owner,
    lf_last_error, lf_destroy,
    LeapfrogNet,
)
from .operators import (  # noqa: F401
    LF_MATRIX_F32, LF_MATRIX_BF16, LF_MATRIX_E4M3, LF_MATRIX_E4M3_128, LF_MATRIX_E4M3_TILES,
    LF_ACT_NONE, LF_ACT_SIGMOID, LF_ACT_RELU, LF_ACT_SILU, LF_ACT_GELU,
    lf_matrix, lf_checkpoint_save, lf_checkpoint_load, lf_norm_forward, lf_norm_workspace_bytes, lf_norm_backward,
    lf_linear_workspace_bytes, lf_linear_forward, lf_linear_backward_workspace_bytes, lf_linear_backward,
    lf_layer_norm_forward, lf_layer_norm_workspace_bytes, lf_layer_norm_backward,
    lf_block_save, lf_block_load, lf_block_linear_workspace_bytes, lf_block_linear_forward,
    lf_block_linear_backward_workspace_bytes, lf_block_linear_backward, lf_distil,
    lf_operator_error,
    E4M3Matrix, E4M3Blocks, RmsNorm, LayerNorm, Linear, BlockLinear, Distillation,
)
from .residual_net import ResidualNet  # noqa: F401
