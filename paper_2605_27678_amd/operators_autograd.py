"""The operators of a cross-attention layer as differentiable PyTorch operations, on torch's current stream: rotary,
gated_norm and cross_attention around the library's calls of operators.py, which move and compute every element.
Gradients are the library's own; they are not differentiable in turn (a second backward raises).

    ranges = torch.from_numpy(hp.hp_image_ranges(token_map)).to(device)      # which states each position sees
    q, = hp.rotary([q], table, positions)
    out = hp.cross_attention(q, k, v, ranges)
    h, z = hp.gated_norm(x, out @ wo, w_post, gate, w_pre, gate_tanh=True)
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

from . import operators as ops
from .autograd import _current_stream


def _rows(t):
    """`t` with its last dimension contiguous, as the calls take it (gradients come in any layout)."""
    return t if t is None or t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


def _scratch(n: int, like):
    return torch.empty(n, dtype=torch.uint8, device=like.device) if n else None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, positions, interleaved, sections, *xs):
        ctx.how = dict(interleaved=interleaved, sections=sections)
        ctx.save_for_backward(table, positions)
        return tuple(_turn(xs, table, positions, False, ctx.how))

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        table, positions = ctx.saved_tensors
        return (None, None, None, None, *_turn(grads, table, positions, True, ctx.how))


def _turn(xs, table, positions, inverse, how):
    xs = [_rows(x) for x in xs]
    outs = [torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in xs]
    ops.hp_rotary(xs, outs, table, positions, inverse=inverse, stream=_current_stream(), **how)
    return outs


def rotary(xs: Sequence[torch.Tensor], table: torch.Tensor, positions: torch.Tensor, *, interleaved: bool = False,
           sections: Optional[Sequence[int]] = None):
    """Every tensor of xs [rows, heads, dim] turned by `positions` (see hp_rotary), as a tuple of new tensors."""
    return _Rotary.apply(table, positions, interleaved, None if sections is None else tuple(sections), *xs)


class _GatedNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, how, x, y, w_post, gate, w_pre):
        x, y = _rows(x), _rows(y)
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        z = None if w_pre is None else torch.empty_like(h)
        rstd = torch.empty(2, x.shape[0], dtype=torch.float32, device=x.device)
        ops.hp_gated_norm(x, y, h, z, w_post, gate, w_pre, rstd=rstd, stream=_current_stream(), **how)
        ctx.how = how
        ctx.save_for_backward(x, y, w_post, gate, w_pre, rstd)
        ctx.set_materialize_grads(False)
        return h, z

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dz):
        x, y, w_post, gate, w_pre, rstd = ctx.saved_tensors
        if dh is None and dz is None:
            return (None,) * 6
        want = [t if t is not None and n else None for t, n in zip((x, y, w_post, gate, w_pre), ctx.needs_input_grad[1:])]
        out = [None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in want]
        sums = any(t is not None for t in out[2:])
        ws = _scratch(ops.hp_gated_norm_workspace(*x.shape), x) if sums else None
        ops.hp_gated_norm_backward(_rows(dh), _rows(dz), x, y, rstd, w_post, gate, w_pre, *out, workspace=ws,
                                   stream=_current_stream(), **ctx.how)
        return (None, *out)


def gated_norm(x, y, w_post=None, gate=None, w_pre=None, *, gate_tanh: bool = False, residual_scale: float = 1.0,
               unit_offset: bool = False, eps: float = 1e-6):
    """(h, z) of hp_gated_norm as new tensors: the residual stream behind a block with output y, and the next block's
    input (None without w_pre)."""
    how = dict(gate_tanh=gate_tanh, residual_scale=residual_scale, unit_offset=unit_offset, eps=eps)
    return _GatedNorm.apply(how, x, y, w_post, gate, w_pre)


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, ranges, scale):
        q, k, v = _rows(q), _rows(k), _rows(v)
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        ops.hp_cross_attend(q, k, v, ranges, out, lse=lse, scale=scale, stream=_current_stream(),
                            workspace=_scratch(ops.hp_cross_attend_workspace(q, k), q))
        ctx.scale = scale
        ctx.save_for_backward(q, k, v, ranges, out, lse)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, ranges, out, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        ops.hp_cross_attend_backward(q, k, v, ranges, out, lse, _rows(dout), dq, dk, dv, scale=ctx.scale,
                                     stream=_current_stream(),
                                     workspace=_scratch(ops.hp_cross_attend_workspace(q, k, "backward"), q))
        return dq, dk, dv, None, None


def cross_attention(q, k, v, ranges=None, scale: Optional[float] = None):
    """Attention of rows q [rows, heads_q, dim] to states k, v [keys, heads_k, dim] (see hp_cross_attend)."""
    return _CrossAttention.apply(q, k, v, ranges, scale)
