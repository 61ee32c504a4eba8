"""MI355X-native boundary layout transform (forward materialise / backward
route) of heterogeneous-parallel multimodal training: a C-ABI library of HIP
kernels (libhp.so) plus this thin binding."""
from .binding import (HpError, Plan, hp_backward, hp_backward_accumulate, hp_forward, hp_forward_static, hp_zero_image_rows, hp_text_grads, hp_get_option, hp_plan_create,
                      hp_plan_create_batched, hp_plan_create_host, hp_plan_create_joined, hp_plan_tune, hp_probe_stream, hp_probe_stream_ex,
                      hp_forget_tuned_shapes, hp_release_cached_memory, hp_profile_enable, hp_profile_read, hp_set_option, hp_version)
from .operators import (RotaryScaling, hp_cross_attend, hp_cross_attend_backward, hp_cross_attend_step, hp_cross_attend_workspace,
                        hp_gated_norm, hp_gated_norm_backward, hp_gated_norm_workspace, hp_image_ranges, hp_rotary, hp_rotary_table)
from .workloads import Grid, TokenMap


def boundary_transform(plan, src_bufs, text_bufs):
    """The transform as one differentiable PyTorch operation (see autograd.py;
    imported on first use so that host-only users of the plan builder do not
    need torch)."""
    from .autograd import boundary_transform as _impl
    return _impl(plan, src_bufs, text_bufs)


def rotary(xs, table, positions, **how):
    """Rotary positions as a differentiable PyTorch operation (operators_autograd.py, imported on first use)."""
    from .operators_autograd import rotary as _impl
    return _impl(xs, table, positions, **how)


def gated_norm(x, y, w_post=None, gate=None, w_pre=None, **how):
    """Norms around a block with its gate and the residual stream as a differentiable PyTorch operation."""
    from .operators_autograd import gated_norm as _impl
    return _impl(x, y, w_post, gate, w_pre, **how)


def cross_attention(q, k, v, ranges=None, scale=None):
    """Attention to packed encoder states as a differentiable PyTorch operation."""
    from .operators_autograd import cross_attention as _impl
    return _impl(q, k, v, ranges, scale)


__all__ = ["rotary", "gated_norm", "cross_attention", "Grid", "TokenMap", "boundary_transform", "Plan", "HpError", "hp_plan_create", "hp_plan_create_host", "hp_plan_create_batched", "hp_plan_create_joined", "hp_plan_tune", "hp_probe_stream", "hp_probe_stream_ex", "hp_release_cached_memory", "hp_forget_tuned_shapes",
           "hp_forward", "hp_forward_static", "hp_zero_image_rows", "hp_text_grads", "hp_backward", "hp_backward_accumulate", "hp_set_option", "hp_get_option", "hp_profile_enable", "hp_profile_read", "hp_version",
           "RotaryScaling", "hp_rotary_table", "hp_rotary", "hp_gated_norm", "hp_gated_norm_backward", "hp_gated_norm_workspace",
           "hp_cross_attend", "hp_cross_attend_step", "hp_cross_attend_backward", "hp_cross_attend_workspace", "hp_image_ranges"]
