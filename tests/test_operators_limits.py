"""Sizes and layouts that the operators' calls refuse before anything is launched (so without a GPU)."""
import ctypes as C

import pytest

from paper_2605_27678_amd import operators as ops
from paper_2605_27678_amd.binding import HP_EINVAL, HP_ELAYOUT, HP_OK

A = 1 << 20                                       # an address that no refused call looks at


def heads(p=A, row=64, head=8):
    return ops.hp_heads_t(p, row, head)


def attend_args(**kw):
    d = dict(dtype=0, heads_q=8, heads_k=2, dim=64, rows=4, keys=6, scale=0.125, q=heads(), k=heads(), v=heads(), out=heads(), ranges=A, lse=A,
             workspace=A, workspace_bytes=1 << 60, dout=heads(), dq=heads(), dk=heads(), dv=heads())
    return ops.hp_attend_args_t(**{**d, **kw})


def workspace(call, **kw):
    return ops._lib().hp_cross_attend_workspace(C.byref(attend_args(**kw)), call)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_backward_refuses_states_whose_lanes_pass_32_bits(dim):
    """Four lanes a state in bf16, two in binary32; a launch has less than 2^32 of them."""
    L, most = ops._lib(), (1 << 30) - 1024
    for keys in (most + 1, 1 << 30, (1 << 31) - 1025):
        assert L.hp_cross_attend_backward(C.byref(attend_args(keys=keys, dim=dim)), None) == HP_ELAYOUT
        assert workspace(2, keys=keys, dim=dim) == HP_ELAYOUT
        assert workspace(2, keys=keys, dim=dim, dtype=1) > 0
        assert workspace(0, keys=keys, dim=dim) >= 0 and workspace(1, keys=keys, dim=dim) >= 0
    assert workspace(2, keys=most, dim=dim) > 0
    assert L.hp_cross_attend(C.byref(attend_args(keys=1 << 30, dim=dim, rows=0)), None) == HP_OK


def test_the_scratch_memory_of_single_tokens_is_refused_where_the_call_is():
    most = 1 << 23
    for rows, code in ((most, None), (most + 1, HP_ELAYOUT), (1 << 27, HP_ELAYOUT)):
        size = workspace(1, rows=rows)
        assert size >= 0 if code is None else size == code
        if code is not None:
            assert ops._lib().hp_cross_attend_step(C.byref(attend_args(rows=rows)), None) == code
    assert workspace(0, rows=most + 1) >= 0


# ---- norms in place ------------------------------------------------------------------------------------------------

B = 2 * A
NORM = dict(dtype=0, gate_size=1, rows=4, hidden=64, residual_scale=1.0, eps=1e-6, x=A, y=B, x_stride=64, y_stride=80, h=3 * A, z=4 * A,
            h_stride=64, z_stride=64, w_post=5 * A, w_pre=6 * A, rstd=7 * A)


@pytest.mark.parametrize("kw", [dict(h=A, h_stride=65), dict(h=B), dict(z=A, z_stride=128), dict(z=B), dict(h=A, z=B, z_stride=-80),
                                dict(x_stride=0, h=A)])
def test_norm_in_place_goes_by_the_same_strides(kw):
    """A row's result would stand where another row is still to be read."""
    L = ops._lib()
    call = lambda **more: L.hp_gated_norm(C.byref(ops.hp_norm_args_t(**{**NORM, **kw, **more})), None)  # noqa: E731
    assert call() == HP_EINVAL and call(rows=0) == HP_OK


@pytest.mark.parametrize("kw", [dict(dx=A, dx_stride=63), dict(dx=B), dict(dy=A, dy_stride=128), dict(dy=B)])
def test_norm_gradients_in_place_go_by_the_same_strides(kw):
    grads = dict(dh=A, dz=B, dh_stride=64, dz_stride=80, dx=3 * A, dy=4 * A, dx_stride=64, dy_stride=64)
    f = {**NORM, "x": 8 * A, "y": 9 * A}
    L = ops._lib()
    call = lambda **more: L.hp_gated_norm_backward(C.byref(ops.hp_norm_args_t(**{**f, **more})),  # noqa: E731
                                                   C.byref(ops.hp_norm_grads_t(**{**grads, **kw})), None)
    assert call() == HP_EINVAL and call(rows=0) == HP_OK


# ---- rotary in place -----------------------------------------------------------------------------------------------

def rotary_args(x, out, rows, n_heads, **kw):
    a = ops.hp_rotary_args_t(**{**dict(dtype=0, n_tensors=1, dim=64, rot=32, n_axes=1, rows=rows, table=A, table_rows=8, positions=B), **kw})
    a.heads[0], a.x[0], a.out[0] = n_heads, x, out
    return a


@pytest.mark.parametrize("code,x,out,rows,n_heads", [
    (HP_OK, heads(None, 640), heads(None, 64), 0, 3),         # nothing at all, as empty tensors come: no place, so not in place
    (HP_OK, heads(None, 640), heads(None, 64), 4, 0), (HP_OK, heads(A, 640), heads(A, 64), 0, 3), (HP_OK, heads(A, 640), heads(A, 64), 4, 0),
    (HP_EINVAL, heads(A, 640, 64), heads(A, 320, 64), 4, 1), (HP_EINVAL, heads(A, 640, 64), heads(A, 640, 128), 4, 2),
    (HP_EINVAL, heads(A, 640, 64), heads(A, 640, 128), 1, 2)])
def test_rotary_in_place_goes_by_the_strides_that_count(code, x, out, rows, n_heads):
    assert ops._lib().hp_rotary(C.byref(rotary_args(x, out, rows, n_heads)), None) == code
