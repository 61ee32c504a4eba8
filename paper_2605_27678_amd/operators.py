"""Binding of the operators in include/hp_operators.h: rotary positions, norms
with a block's gate and residual stream, and attention to an encoder's states.
Argument marshalling only, same names as the C calls; results go into buffers of
the caller's, on the stream that is passed (None = the default stream), ordered
against that stream only.  operators_autograd.py has the same operators as
differentiable PyTorch operations.

Every buffer is a CUDA tensor of the current device in bfloat16 or float32 (all
of one call's the same) whose last dimension is contiguous; other strides are
taken as they are.  A wrong shape, type or device raises ValueError before
anything is launched, an argument that the library refuses raises HpError."""
from __future__ import annotations

import ctypes as C
import sys
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

from . import binding
from .binding import HpError, _check, _stream_handle, _token_map, hp_token_map_t
from .workloads import TokenMap

MAX_TENSORS = MAX_AXES = 4


class hp_heads_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class hp_rotary_scaling_t(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("base", C.c_double), ("factor", C.c_double),
                ("original_length", C.c_double), ("low_turns", C.c_double), ("high_turns", C.c_double),
                ("amplitude", C.c_double)]


class hp_rotary_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_tensors", C.c_int32), ("dim", C.c_int32), ("rot", C.c_int32),
                ("interleaved", C.c_int32), ("inverse", C.c_int32), ("n_axes", C.c_int32),
                ("sections", C.c_int32 * MAX_AXES), ("reserved", C.c_int32), ("rows", C.c_int64),
                ("table", C.c_void_p), ("table_rows", C.c_int64), ("positions", C.c_void_p),
                ("axis_stride", C.c_int64), ("heads", C.c_int32 * MAX_TENSORS),
                ("x", hp_heads_t * MAX_TENSORS), ("out", hp_heads_t * MAX_TENSORS)]


class hp_norm_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("gate_size", C.c_int32), ("gate_tanh", C.c_int32),
                ("unit_offset", C.c_int32), ("rows", C.c_int64), ("hidden", C.c_int32),
                ("residual_scale", C.c_float), ("eps", C.c_float), ("reserved", C.c_int32),
                ("x", C.c_void_p), ("y", C.c_void_p), ("x_stride", C.c_int64), ("y_stride", C.c_int64),
                ("h", C.c_void_p), ("z", C.c_void_p), ("h_stride", C.c_int64), ("z_stride", C.c_int64),
                ("w_post", C.c_void_p), ("gate", C.c_void_p), ("w_pre", C.c_void_p), ("rstd", C.c_void_p)]


class hp_norm_grads_t(C.Structure):
    _fields_ = [("dh", C.c_void_p), ("dz", C.c_void_p), ("dh_stride", C.c_int64), ("dz_stride", C.c_int64),
                ("dx", C.c_void_p), ("dy", C.c_void_p), ("dx_stride", C.c_int64), ("dy_stride", C.c_int64),
                ("dw_post", C.c_void_p), ("dgate", C.c_void_p), ("dw_pre", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class hp_attend_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_k", C.c_int32), ("dim", C.c_int32),
                ("rows", C.c_int64), ("keys", C.c_int64), ("scale", C.c_float), ("reserved", C.c_int32),
                ("q", hp_heads_t), ("k", hp_heads_t), ("v", hp_heads_t), ("out", hp_heads_t),
                ("ranges", C.c_void_p), ("lse", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64),
                ("dout", hp_heads_t), ("dq", hp_heads_t), ("dk", hp_heads_t), ("dv", hp_heads_t)]


EXPORTS = ["hp_rotary_table", "hp_rotary", "hp_gated_norm", "hp_gated_norm_backward", "hp_gated_norm_workspace",
           "hp_cross_attend", "hp_cross_attend_step", "hp_cross_attend_backward", "hp_cross_attend_workspace",
           "hp_image_ranges"]

_ready = None
_fast = None            # hp_marshal, or False where it is not used
_at = {}                # addresses of the calls that go through it


def _extension():
    """hp_marshal, or False."""
    global _fast
    if _fast is None:
        if "torch" not in sys.modules:
            return False
        if binding._marshal is None:
            binding._load_marshal()
        _fast = binding._marshal_module or False
        L = _lib()
        for f in ("hp_rotary", "hp_gated_norm", "hp_gated_norm_backward", "hp_cross_attend", "hp_cross_attend_step",
                  "hp_cross_attend_backward"):
            _at[f] = C.cast(getattr(L, f), C.c_void_p).value
    return _fast


def _call(function: str, name: str, *args) -> bool:
    """The call through hp_marshal.  False if the arguments need a closer look than it takes."""
    if not _extension():
        return False
    rc = getattr(_fast, function)(_at[name], *args)
    if rc is None:
        return False
    if rc < 0:
        raise HpError(rc, name)
    return True


def _lib():
    global _ready
    if _ready is not None:
        return _ready
    L = binding._lib()
    p, i32, i64 = C.POINTER, C.c_int32, C.c_int64
    L.hp_rotary_table.argtypes = [C.c_void_p, i64, i64, i32, p(hp_rotary_scaling_t), C.c_void_p]
    L.hp_rotary.argtypes = [p(hp_rotary_args_t), C.c_void_p]
    L.hp_gated_norm.argtypes = [p(hp_norm_args_t), C.c_void_p]
    L.hp_gated_norm_backward.argtypes = [p(hp_norm_args_t), p(hp_norm_grads_t), C.c_void_p]
    L.hp_gated_norm_workspace.argtypes = [i64, i32]
    L.hp_gated_norm_workspace.restype = i64
    for f in ("hp_cross_attend", "hp_cross_attend_step", "hp_cross_attend_backward"):
        getattr(L, f).argtypes = [p(hp_attend_args_t), C.c_void_p]
    L.hp_cross_attend_workspace.argtypes = [p(hp_attend_args_t), i32]
    L.hp_cross_attend_workspace.restype = i64
    L.hp_image_ranges.argtypes = [p(hp_token_map_t), i32, p(i32)]
    _ready = L
    return L


def _dtype(t) -> int:
    torch = sys.modules["torch"]
    if t.dtype is torch.bfloat16:
        return 0
    if t.dtype is torch.float32:
        return 1
    raise ValueError(f"need bfloat16 or float32 tensors, got {t.dtype}")


def _tensor(t, what: str, shape, dtype=None, like=None, contiguous=False):
    """`t` as it is, if it is a CUDA tensor of the current device with this shape (None: any size there)."""
    torch = sys.modules.get("torch")
    if torch is None or not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what}: need a CUDA tensor")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what}: on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    if t.dim() != len(shape) or any(n is not None and m != n for m, n in zip(t.shape, shape)):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, need {tuple('any' if n is None else n for n in shape)}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{what}: need {dtype}, got {t.dtype}")
    if like is not None and t.dtype is not like.dtype:
        raise ValueError(f"{what}: {t.dtype} beside {like.dtype}")
    if contiguous:
        if not t.is_contiguous():
            raise ValueError(f"{what}: need a contiguous tensor")
    elif t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the last dimension has to be contiguous")
    return t


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() else None


def _heads(t) -> hp_heads_t:
    return hp_heads_t(_ptr(t), t.stride(0), t.stride(1))


def _scratch(t, what: str = "workspace"):
    """(pointer, bytes) of scratch memory: any contiguous CUDA tensor, or None."""
    if t is None:
        return None, 0
    _tensor(t, what, (None,) * t.dim(), contiguous=True)
    return _ptr(t), t.numel() * t.element_size()


# ---- rotary positions ------------------------------------------------------------------------------------

@dataclass(frozen=True)
class RotaryScaling:
    """How frequencies are stretched for sequences longer than the model was trained on: `kind` "plain", "linear"
    (divided by factor), "base" (the base grows so that the lowest is divided by factor) or "by_turns" (divided where
    a pair turns at most low_turns times over original_length positions, kept from high_turns on, linear between);
    `amplitude` multiplies cosines and sines."""
    kind: str = "plain"
    factor: float = 1.0
    original_length: float = 0.0
    low_turns: float = 1.0
    high_turns: float = 32.0
    amplitude: float = 1.0


SCALINGS = {"plain": 0, "linear": 1, "base": 2, "by_turns": 3}


def hp_rotary_table(table, base: float = 10000.0, scaling: Optional[RotaryScaling] = None, first: int = 0,
                    stream=None) -> None:
    """Fills table, float32 [positions, rot / 2, 2], with the cosines and sines of positions first, first + 1, .."""
    torch = sys.modules.get("torch")
    s = scaling or RotaryScaling()
    if s.kind not in SCALINGS:
        raise ValueError(f"scaling {s.kind!r}: one of {', '.join(SCALINGS)}")
    _tensor(table, "table", (None, None, 2), dtype=torch.float32 if torch else None, contiguous=True)
    arg = hp_rotary_scaling_t(SCALINGS[s.kind], 0, float(base), s.factor, s.original_length, s.low_turns, s.high_turns,
                              s.amplitude)
    _check(_lib().hp_rotary_table(_ptr(table), table.shape[0], int(first), 2 * table.shape[1], C.byref(arg),
                                  _stream_handle(stream)), "hp_rotary_table")


def hp_rotary(xs: Sequence, outs: Sequence, table, positions, *, interleaved: bool = False, inverse: bool = False,
              sections: Optional[Sequence[int]] = None, stream=None) -> None:
    """outs[t] = xs[t] [rows, heads, dim] turned by `positions`, int32 [rows], or [axes, rows] with `sections`, the
    numbers of pairs that go by each axis.  The table's width says how many channels turn.  xs and outs: lists of up
    to four tensors (queries and keys); an output may be its input."""
    if _call("rotary", "hp_rotary", xs, outs, table, positions, interleaved, inverse, sections, stream):
        return
    torch = sys.modules.get("torch")
    if not 1 <= len(xs) <= MAX_TENSORS or len(xs) != len(outs):
        raise ValueError(f"need 1 to {MAX_TENSORS} tensors and as many outputs")
    a = hp_rotary_args_t()
    rows, dim = None, None
    for i, (x, o) in enumerate(zip(xs, outs)):
        _tensor(x, f"xs[{i}]", (rows, None, dim), like=xs[0])
        rows, dim = x.shape[0], x.shape[2]
        _tensor(o, f"outs[{i}]", x.shape, like=x)
        a.heads[i] = x.shape[1]
        a.x[i], a.out[i] = _heads(x), _heads(o)
    _tensor(table, "table", (None, None, 2), dtype=torch.float32, contiguous=True)
    if sections is None:
        _tensor(positions, "positions", (rows,), dtype=torch.int32)
        a.n_axes = 1
    else:
        if not 1 <= len(sections) <= MAX_AXES or sum(sections) != table.shape[1]:
            raise ValueError(f"sections: 1 to {MAX_AXES} of them, {table.shape[1]} pairs in all")
        _tensor(positions, "positions", (len(sections), rows), dtype=torch.int32)
        a.n_axes, a.axis_stride = len(sections), positions.stride(0)
        a.sections[:len(sections)] = [int(n) for n in sections]
    a.dtype, a.n_tensors, a.dim, a.rot = _dtype(xs[0]), len(xs), dim, 2 * table.shape[1]
    a.interleaved, a.inverse, a.rows = bool(interleaved), bool(inverse), rows
    a.table, a.table_rows, a.positions = _ptr(table), table.shape[0], _ptr(positions)
    _check(_lib().hp_rotary(C.byref(a), _stream_handle(stream)), "hp_rotary")


# ---- norms around a block, its gate and the residual stream -------------------------------------------------

def _norm_args(x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset, eps, rstd) -> hp_norm_args_t:
    torch = sys.modules.get("torch")
    _tensor(x, "x", (None, None))
    rows, hidden = x.shape
    a = hp_norm_args_t(dtype=_dtype(x), rows=rows, hidden=hidden, residual_scale=residual_scale, eps=eps,
                       gate_tanh=bool(gate_tanh), unit_offset=bool(unit_offset), x=_ptr(x), x_stride=x.stride(0))
    if y is not None:
        _tensor(y, "y", (rows, hidden), like=x)
        a.y, a.y_stride = _ptr(y), y.stride(0)
    for name, w in (("w_post", w_post), ("w_pre", w_pre)):
        if w is not None:
            setattr(a, name, _ptr(_tensor(w, name, (hidden,), like=x, contiguous=True)))
    if gate is not None:
        _tensor(gate, "gate", (None,), like=x, contiguous=True)
        if not gate.numel():                             # its address would be that of no gate
            raise ValueError("gate: no values, need one or one a channel")
        a.gate, a.gate_size = _ptr(gate), gate.numel()
    if rstd is not None:
        a.rstd = _ptr(_tensor(rstd, "rstd", (2, rows), dtype=torch.float32, contiguous=True))
    return a


def hp_gated_norm(x, y, h, z, w_post=None, gate=None, w_pre=None, *, gate_tanh: bool = False,
                  residual_scale: float = 1.0, unit_offset: bool = False, eps: float = 1e-6, rstd=None,
                  stream=None) -> None:
    """h = residual_scale * x + t * norm(y) * w_post and z = norm(h) * w_pre for rows [rows, hidden]; t = gate or
    tanh(gate), one value or one a channel.  w_post None: y is taken as it is; gate None: t = 1; y None: no block.
    h or z None: not written.  rstd: float32 [2, rows] for the backward call."""
    if _call("norm", "hp_gated_norm", x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset, eps, rstd, h, z,
             stream):
        return
    a = _norm_args(x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset, eps, rstd)
    for name, t in (("h", h), ("z", z)):
        if t is not None:
            setattr(a, name, _ptr(_tensor(t, name, x.shape, like=x)))
            setattr(a, name + "_stride", t.stride(0))
    _check(_lib().hp_gated_norm(C.byref(a), _stream_handle(stream)), "hp_gated_norm")


def hp_gated_norm_workspace(rows: int, hidden: int) -> int:
    """Bytes of scratch memory that hp_gated_norm_backward needs for the gradients of weights and gate."""
    return _check(_lib().hp_gated_norm_workspace(int(rows), int(hidden)), "hp_gated_norm_workspace")


def hp_gated_norm_backward(dh, dz, x, y, rstd, w_post, gate, w_pre, dx, dy, dw_post, dgate, dw_pre, *,
                           gate_tanh: bool = False, residual_scale: float = 1.0, unit_offset: bool = False,
                           eps: float = 1e-6, workspace=None, stream=None) -> None:
    """Gradients of hp_gated_norm from those of h and z (one may be None).  Outputs that are None are not computed."""
    if _call("norm_backward", "hp_gated_norm_backward", x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset,
             eps, rstd, dh, dz, dx, dy, dw_post, dgate, dw_pre, workspace, stream):
        return
    a = _norm_args(x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset, eps, rstd)
    g = hp_norm_grads_t()
    for name, t in (("dh", dh), ("dz", dz), ("dx", dx), ("dy", dy)):
        if t is not None:
            setattr(g, name, _ptr(_tensor(t, name, x.shape, like=x)))
            setattr(g, name + "_stride", t.stride(0))
    for name, t, w in (("dw_post", dw_post, w_post), ("dgate", dgate, gate), ("dw_pre", dw_pre, w_pre)):
        if t is not None:
            if w is None:
                raise ValueError(f"{name}: there is nothing that it is the gradient of")
            setattr(g, name, _ptr(_tensor(t, name, w.shape, like=x, contiguous=True)))
    g.workspace, g.workspace_bytes = _scratch(workspace)
    _check(_lib().hp_gated_norm_backward(C.byref(a), C.byref(g), _stream_handle(stream)), "hp_gated_norm_backward")


# ---- cross attention ------------------------------------------------------------------------------------------

CALLS = {"forward": 0, "step": 1, "backward": 2}


def _attend_args(q, k, v, ranges, out, lse, scale, workspace) -> hp_attend_args_t:
    torch = sys.modules.get("torch")
    _tensor(q, "q", (None, None, None))
    rows, heads_q, dim = q.shape
    _tensor(k, "k", (None, None, dim), like=q)
    keys, heads_k, _ = k.shape
    _tensor(v, "v", k.shape, like=q)
    _tensor(out, "out", q.shape, like=q)
    a = hp_attend_args_t(dtype=_dtype(q), heads_q=heads_q, heads_k=heads_k, dim=dim, rows=rows, keys=keys,
                         scale=dim ** -0.5 if scale is None else scale, q=_heads(q), k=_heads(k), v=_heads(v),
                         out=_heads(out))
    if ranges is not None:
        a.ranges = _ptr(_tensor(ranges, "ranges", (rows, 2), dtype=torch.int32, contiguous=True))
    if lse is not None:
        a.lse = _ptr(_tensor(lse, "lse", (rows, heads_q), dtype=torch.float32, contiguous=True))
    a.workspace, a.workspace_bytes = _scratch(workspace)
    return a


def hp_cross_attend(q, k, v, ranges, out, *, lse=None, scale: Optional[float] = None, workspace=None,
                    stream=None) -> None:
    """out = attention of query rows q [rows, heads_q, dim] to states k, v [keys, heads_k, dim]; row r sees states
    ranges[r, 0] to ranges[r, 1] - 1 (int32; None: all).  scale None: 1 / sqrt(dim).  lse: float32 [rows, heads_q]
    for the backward call."""
    if _call("attend", "hp_cross_attend", q, k, v, ranges, out, lse, scale, workspace, None, stream):
        return
    a = _attend_args(q, k, v, ranges, out, lse, scale, workspace)
    _check(_lib().hp_cross_attend(C.byref(a), _stream_handle(stream)), "hp_cross_attend")


def hp_cross_attend_step(q, k, v, ranges, out, *, lse=None, scale: Optional[float] = None, workspace=None,
                         stream=None) -> None:
    """hp_cross_attend for rows that share nothing, as single tokens of many requests."""
    if _call("attend", "hp_cross_attend_step", q, k, v, ranges, out, lse, scale, workspace, None, stream):
        return
    a = _attend_args(q, k, v, ranges, out, lse, scale, workspace)
    _check(_lib().hp_cross_attend_step(C.byref(a), _stream_handle(stream)), "hp_cross_attend_step")


def hp_cross_attend_backward(q, k, v, ranges, out, lse, dout, dq, dk, dv, *, scale: Optional[float] = None,
                             workspace=None, stream=None) -> None:
    """Gradients of q, k and v from the forward's arguments, its out and lse, and the gradient of out."""
    if _call("attend", "hp_cross_attend_backward", q, k, v, ranges, out, lse, scale, workspace, (dout, dq, dk, dv), stream):
        return
    a = _attend_args(q, k, v, ranges, out, lse, scale, workspace)
    for name, t, like in (("dout", dout, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, k)):
        setattr(a, name, _heads(_tensor(t, name, like.shape, like=q)))
    _check(_lib().hp_cross_attend_backward(C.byref(a), _stream_handle(stream)), "hp_cross_attend_backward")


def hp_cross_attend_workspace(q, k, call: str = "forward") -> int:
    """Bytes of scratch memory that a call ("forward", "step" or "backward") needs for tensors of these shapes."""
    if call not in CALLS:
        raise ValueError(f"call {call!r}: one of {', '.join(CALLS)}")
    a = hp_attend_args_t(dtype=_dtype(q), heads_q=q.shape[1], heads_k=k.shape[1], dim=q.shape[2], rows=q.shape[0],
                         keys=k.shape[0])
    return _check(_lib().hp_cross_attend_workspace(C.byref(a), CALLS[call]), "hp_cross_attend_workspace")


RULES = {"sample": 0, "previous": 1, "latest": 2}


def hp_image_ranges(tmap: TokenMap, rule: str = "previous") -> np.ndarray:
    """int32 [batch * seq, 2]: the rows of the packed image tokens that each position sees - every image of its sample,
    those that end at or before it, or the latest of these."""
    if rule not in RULES:
        raise ValueError(f"rule {rule!r}: one of {', '.join(RULES)}")
    t, keep = _token_map(tmap)
    out = np.zeros((max(tmap.batch, 0) * max(tmap.seq, 0), 2), np.int32)
    _check(_lib().hp_image_ranges(C.byref(t), RULES[rule], out.ctypes.data_as(C.POINTER(C.c_int32))), "hp_image_ranges")
    del keep
    return out
