"""Binding of include/hp_packed.h: states and weights held in 4 bits.  Argument marshalling only, as in operators.py,
whose rules for tensors, streams and errors hold here too.

    cache_k, cache_v = (hp.Packed.room(rows, heads_k, dim, device) for _ in range(2))
    hp.hp_pack([k, v], [cache_k.rows(a, b), cache_v.rows(a, b)])       # as a request's states are made
    hp.hp_packed_attend_step(q, cache_k, cache_v, ranges, out, workspace=scratch)
    hp.hp_packed_linear(x, w, y)                                       # y = x w^T
"""
from __future__ import annotations

import ctypes as C
import sys
from typing import NamedTuple, Optional, Sequence

from . import binding, operators
from .binding import HpError, _check, _stream_handle
from .operators import _dtype, _heads, _ptr, _scratch, _tensor, hp_heads_t

GROUP = 32
MAX_TENSORS = 4


class hp_packed_t(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("code_row_stride", C.c_int64), ("code_head_stride", C.c_int64),
                ("scale_row_stride", C.c_int64), ("scale_head_stride", C.c_int64)]


class hp_pack_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_tensors", C.c_int32), ("dim", C.c_int32), ("reserved", C.c_int32), ("rows", C.c_int64),
                ("heads", C.c_int32 * MAX_TENSORS), ("x", hp_heads_t * MAX_TENSORS), ("packed", hp_packed_t * MAX_TENSORS)]


class hp_packed_attend_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_k", C.c_int32), ("dim", C.c_int32), ("rows", C.c_int64),
                ("keys", C.c_int64), ("scale", C.c_float), ("reserved", C.c_int32), ("q", hp_heads_t), ("out", hp_heads_t),
                ("k", hp_packed_t), ("v", hp_packed_t), ("ranges", C.c_void_p), ("lse", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64)]


class hp_packed_linear_args_t(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_in", C.c_int32), ("n_out", C.c_int32), ("reserved", C.c_int32), ("rows", C.c_int64),
                ("x", C.c_void_p), ("x_stride", C.c_int64), ("w", hp_packed_t), ("out", C.c_void_p), ("out_stride", C.c_int64)]


EXPORTS = ["hp_pack", "hp_unpack", "hp_packed_attend_step", "hp_packed_attend_workspace", "hp_packed_linear"]


class Packed(NamedTuple):
    """Packed rows: codes, uint8 [rows, heads, 16 * groups], and scales, bfloat16 [rows, heads, groups, 2] (step, low); a
    matrix has no heads.  Any pair of tensors of these shapes will do where a Packed is asked for."""
    codes: "torch.Tensor"            # noqa: F821
    scales: "torch.Tensor"           # noqa: F821

    @classmethod
    def room(cls, rows: int, heads: Optional[int], dim: int, device) -> "Packed":
        """Memory for packed rows, the rows of a head one behind the other; heads None: a matrix's."""
        torch = sys.modules["torch"]
        g = (dim + GROUP - 1) // GROUP
        lead = (rows,) if heads is None else (heads, rows)
        codes = torch.empty(*lead, 16 * g, dtype=torch.uint8, device=device)
        scales = torch.empty(*lead, g, 2, dtype=torch.bfloat16, device=device)
        return cls(codes, scales) if heads is None else cls(codes.transpose(0, 1), scales.transpose(0, 1))

    def rows(self, first: int, end: int) -> "Packed":
        """Rows first to end - 1, as a view."""
        return Packed(self.codes[first:end], self.scales[first:end])


_ready = None
_at = {}


def _lib():
    global _ready
    if _ready is not None:
        return _ready
    L = binding._lib()
    p = C.POINTER
    for f in ("hp_pack", "hp_unpack"):
        getattr(L, f).argtypes = [p(hp_pack_args_t), C.c_void_p]
    L.hp_packed_attend_step.argtypes = [p(hp_packed_attend_args_t), C.c_void_p]
    L.hp_packed_attend_workspace.argtypes = [p(hp_packed_attend_args_t)]
    L.hp_packed_attend_workspace.restype = C.c_int64
    L.hp_packed_linear.argtypes = [p(hp_packed_linear_args_t), C.c_void_p]
    for f in ("hp_pack", "hp_unpack", "hp_packed_attend_step", "hp_packed_linear"):
        _at[f] = C.cast(getattr(L, f), C.c_void_p).value
    _ready = L
    return L


def _call(function: str, name: str, *args) -> bool:
    """The call through hp_marshal.  False if the arguments need a closer look than it takes."""
    fast = operators._extension()
    if not fast:
        return False
    _lib()
    rc = getattr(fast, function)(_at[name], *args)
    if rc is None:
        return False
    if rc < 0:
        raise HpError(rc, name)
    return True


MATRIX = "matrix"           # in the place of a number of heads


def _packed(t, what: str, rows, heads, dim) -> hp_packed_t:
    """The pair `t` as the C ABI takes it: `rows` rows (None: any) of `heads` heads (None: any) and `dim` channels."""
    torch = sys.modules.get("torch")
    if not isinstance(t, (tuple, list)) or len(t) != 2:
        raise ValueError(f"{what}: need codes and scales")
    g = (dim + GROUP - 1) // GROUP
    lead = (rows,) if heads == MATRIX else (rows, heads)
    codes = _tensor(t[0], f"{what} codes", (*lead, 16 * g), dtype=torch.uint8 if torch else None)
    scales = _tensor(t[1], f"{what} scales", (*lead, g, 2), dtype=torch.bfloat16 if torch else None)
    if codes.shape[:-1] != scales.shape[:-2]:
        raise ValueError(f"{what}: codes of {tuple(codes.shape[:-1])} rows, scales of {tuple(scales.shape[:-2])}")
    if g > 1 and scales.stride(-2) != 2:
        raise ValueError(f"{what} scales: a row's groups have to be contiguous")
    a = hp_packed_t(_ptr(codes), _ptr(scales), codes.stride(0), 0, scales.stride(0), 0)
    if heads != MATRIX:
        a.code_head_stride, a.scale_head_stride = codes.stride(1), scales.stride(1)
    return a


def _pack_args(xs, packed) -> hp_pack_args_t:
    if not 1 <= len(xs) <= MAX_TENSORS or len(xs) != len(packed):
        raise ValueError(f"need 1 to {MAX_TENSORS} tensors and as many packed ones")
    a = hp_pack_args_t(n_tensors=len(xs))
    rows, dim = None, None
    for i, (x, t) in enumerate(zip(xs, packed)):
        matrix = getattr(x, "ndim", 3) == 2
        _tensor(x, f"xs[{i}]", (rows, dim) if matrix else (rows, None, dim), like=xs[0])
        rows, dim = x.shape[0], x.shape[-1]
        a.heads[i] = 1 if matrix else x.shape[1]
        a.x[i] = hp_heads_t(_ptr(x), x.stride(0), 0 if matrix else x.stride(1))
        a.packed[i] = _packed(t, f"packed[{i}]", rows, MATRIX if matrix else x.shape[1], dim)
    a.dtype, a.rows, a.dim = _dtype(xs[0]), rows, dim
    return a


def hp_pack(xs: Sequence, packed: Sequence, *, stream=None) -> None:
    """packed[t] = xs[t], up to four tensors [rows, heads, dim] (or matrices [rows, dim]) of the same rows and dim."""
    if _call("pack", "hp_pack", xs, packed, stream):
        return
    _check(_lib().hp_pack(C.byref(_pack_args(xs, packed)), _stream_handle(stream)), "hp_pack")


def hp_unpack(packed: Sequence, outs: Sequence, *, stream=None) -> None:
    """outs[t] = the values of packed[t], up to four tensors [rows, heads, dim] (or matrices [rows, dim])."""
    if _call("pack", "hp_unpack", outs, packed, stream):
        return
    _check(_lib().hp_unpack(C.byref(_pack_args(outs, packed)), _stream_handle(stream)), "hp_unpack")


def hp_packed_attend_step(q, k, v, ranges, out, *, lse=None, scale: Optional[float] = None, workspace=None, stream=None) -> None:
    """hp_cross_attend_step with k and v Packed: out = attention of single tokens q [rows, heads_q, dim] to packed states
    [keys, heads_k, dim]; row r sees states ranges[r, 0] to ranges[r, 1] - 1 (int32; None: all).  scale None: 1 / sqrt(dim)."""
    if _call("packed_attend", "hp_packed_attend_step", q, k, v, ranges, out, lse, scale, workspace, stream):
        return
    torch = sys.modules.get("torch")
    _tensor(q, "q", (None, None, None))
    rows, heads_q, dim = q.shape
    _tensor(out, "out", q.shape, like=q)
    a = hp_packed_attend_args_t(dtype=_dtype(q), heads_q=heads_q, dim=dim, rows=rows, scale=dim ** -0.5 if scale is None else scale,
                                q=_heads(q), out=_heads(out), k=_packed(k, "k", None, None, dim))
    a.keys, a.heads_k = k[0].shape[0], k[0].shape[1]
    a.v = _packed(v, "v", a.keys, a.heads_k, dim)
    if ranges is not None:
        a.ranges = _ptr(_tensor(ranges, "ranges", (rows, 2), dtype=torch.int32, contiguous=True))
    if lse is not None:
        a.lse = _ptr(_tensor(lse, "lse", (rows, heads_q), dtype=torch.float32, contiguous=True))
    a.workspace, a.workspace_bytes = _scratch(workspace)
    _check(_lib().hp_packed_attend_step(C.byref(a), _stream_handle(stream)), "hp_packed_attend_step")


def hp_packed_attend_workspace(q, k) -> int:
    """Bytes of scratch memory that hp_packed_attend_step needs for q and packed states k of these shapes."""
    a = hp_packed_attend_args_t(dtype=_dtype(q), heads_q=q.shape[1], heads_k=k[0].shape[1], dim=q.shape[2], rows=q.shape[0], keys=k[0].shape[0])
    return _check(_lib().hp_packed_attend_workspace(C.byref(a)), "hp_packed_attend_workspace")


def hp_packed_linear(x, w, out, *, stream=None) -> None:
    """out [rows, n_out] = x [rows, n_in] times the transpose of w, Packed [n_out, n_in]."""
    if _call("packed_linear", "hp_packed_linear", x, w, out, stream):
        return
    _tensor(x, "x", (None, None))
    rows, n_in = x.shape
    a = hp_packed_linear_args_t(dtype=_dtype(x), n_in=n_in, rows=rows, x=_ptr(x), x_stride=x.stride(0), w=_packed(w, "w", None, MATRIX, n_in))
    a.n_out = w[0].shape[0]
    _tensor(out, "out", (rows, a.n_out), like=x)
    a.out, a.out_stride = _ptr(out), out.stride(0)
    _check(_lib().hp_packed_linear(C.byref(a), _stream_handle(stream)), "hp_packed_linear")
