"""The operators' host side: what the calls refuse (before any HIP call, so without a GPU), scratch sizes, image ranges,
and the two headers against the binding."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paper_2605_27678_amd as hp
from paper_2605_27678_amd import operators as ops
from paper_2605_27678_amd import workloads as wl
from paper_2605_27678_amd.binding import HP_EALIGN, HP_EINVAL, HP_ELAYOUT, HP_EMAP, HP_OK, HpError

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                       # an address that no refused call looks at


def heads(p=A, row=64, head=8):
    return ops.hp_heads_t(p, row, head)


def test_the_header_declares_what_the_binding_has():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hp_operators.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(hp_\w+)\s*\(", text)) == set(ops.EXPORTS)
    for name in ops.EXPORTS:
        assert getattr(ops._lib(), name) and name in hp.__all__


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++11")])
def test_the_header_is_plain_c_and_its_structs_are_the_bindings(compiler, std, tmp_path):
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    names = ["hp_heads_t", "hp_rotary_scaling_t", "hp_rotary_args_t", "hp_norm_args_t", "hp_norm_grads_t", "hp_attend_args_t"]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hp_operators.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", sizeof({n}));\n' for n in names) +
                   "".join(f'  printf("%zu\\n", offsetof({n}, {f}));\n' for n in names for f, *_ in getattr(ops, n)._fields_) +
                   "  return 0; }\n")
    exe = tmp_path / "t"
    subprocess.run([compiler, std, "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe)], check=True, capture_output=True, timeout=120)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, timeout=30).stdout.split()]
    structs = [getattr(ops, n) for n in names]
    assert got == [C.sizeof(s) for s in structs] + [getattr(s, f).offset for s in structs for f, *_ in s._fields_]


# ---- rotary ------------------------------------------------------------------------------------------------------

def rotary_args(**kw):
    a = ops.hp_rotary_args_t(dtype=0, n_tensors=2, dim=64, rot=32, n_axes=1, rows=4, table=A, table_rows=8, positions=A)
    for t in range(2):
        a.heads[t], a.x[t], a.out[t] = 3, heads(), heads(2 * A)
    for n, v in kw.items():
        if "_at_" in n:
            getattr(a, n.split("_at_")[0])[int(n[-1])] = v
        elif n == "sections":
            a.sections[:len(v)] = v
        else:
            setattr(a, n, v)
    return a


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(dtype=2)), (HP_EINVAL, dict(n_tensors=0)), (HP_EINVAL, dict(n_tensors=5)), (HP_EINVAL, dict(rows=-1)),
    (HP_EINVAL, dict(rot=0)), (HP_EINVAL, dict(rot=31)), (HP_EINVAL, dict(rot=66)), (HP_EINVAL, dict(dim=1)), (HP_EINVAL, dict(dim=1025)),
    (HP_EINVAL, dict(table_rows=0)), (HP_EINVAL, dict(table=None)), (HP_EINVAL, dict(positions=None)), (HP_EINVAL, dict(n_axes=0)),
    (HP_EINVAL, dict(n_axes=5)), (HP_EINVAL, dict(n_axes=2, sections=[8, 7])), (HP_EINVAL, dict(n_axes=2, sections=[8, 9])),
    (HP_EINVAL, dict(n_axes=2, sections=[17, -1])), (HP_EINVAL, dict(x_at_1=heads(None))), (HP_EINVAL, dict(out_at_0=heads(None))),
    (HP_EINVAL, dict(heads_at_0=-1)), (HP_EINVAL, dict(heads_at_0=4097)), (HP_EINVAL, dict(out_at_0=heads(A, 65))),
    (HP_EALIGN, dict(x_at_0=heads(A + 1))), (HP_EALIGN, dict(out_at_1=heads(A + 1))), (HP_EALIGN, dict(dtype=1, x_at_0=heads(A + 2))),
    (HP_EALIGN, dict(table=A + 2)), (HP_EALIGN, dict(positions=A + 2)),
    (HP_OK, dict(rows=0)), (HP_OK, dict(heads_at_0=0, heads_at_1=0)), (HP_OK, dict(rows=0, x_at_0=heads(None)))])
def test_rotary_refuses(code, kw):
    assert ops._lib().hp_rotary(C.byref(rotary_args(**kw)), None) == code


def test_rotary_refuses_no_arguments():
    L = ops._lib()
    assert L.hp_rotary(None, None) == HP_EINVAL
    assert L.hp_rotary_table(A, 4, 0, 32, None, None) == HP_EINVAL


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(n=-1)), (HP_EINVAL, dict(first=-1)), (HP_EINVAL, dict(rot=3)), (HP_EINVAL, dict(rot=0)), (HP_EINVAL, dict(table=None)),
    (HP_EINVAL, dict(kind=4)), (HP_EINVAL, dict(base=0.0)), (HP_EINVAL, dict(base=float("nan"))), (HP_EINVAL, dict(kind=1, factor=0.0)),
    (HP_EINVAL, dict(kind=1, factor=float("inf"))), (HP_EINVAL, dict(kind=2, factor=2.0, rot=2)), (HP_EINVAL, dict(kind=3, factor=2.0)),
    (HP_EINVAL, dict(kind=3, factor=2.0, original_length=100.0, low_turns=4.0, high_turns=4.0)), (HP_EINVAL, dict(amplitude=float("inf"))),
    (HP_EALIGN, dict(table=A + 2)), (HP_OK, dict(n=0)), (HP_OK, dict(n=0, table=None))])
def test_rotary_table_refuses(code, kw):
    at = dict(table=A, n=4, first=0, rot=32)
    at.update({n: kw.pop(n) for n in list(kw) if n in at})
    s = ops.hp_rotary_scaling_t(**{**dict(kind=0, base=10000.0, amplitude=1.0), **kw})
    assert ops._lib().hp_rotary_table(at["table"], at["n"], at["first"], at["rot"], C.byref(s), None) == code


# ---- norm ----------------------------------------------------------------------------------------------------------

NORM = dict(dtype=0, gate_size=64, rows=4, hidden=64, residual_scale=1.0, eps=1e-6, x=A, y=A, x_stride=64, y_stride=64, h=A, z=A,
            h_stride=64, z_stride=64, w_post=A, gate=A, w_pre=A, rstd=A)


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(dtype=-1)), (HP_EINVAL, dict(rows=-1)), (HP_EINVAL, dict(hidden=0)), (HP_EINVAL, dict(hidden=32769, gate_size=1)),
    (HP_EINVAL, dict(gate_size=2)), (HP_EINVAL, dict(eps=-1.0)), (HP_EINVAL, dict(eps=float("nan"))), (HP_EINVAL, dict(residual_scale=float("inf"))),
    (HP_EINVAL, dict(x=None)), (HP_EINVAL, dict(y=None)), (HP_EINVAL, dict(y=None, w_post=None)), (HP_EINVAL, dict(h=None, z=None)),
    (HP_EINVAL, dict(w_pre=None)), (HP_EALIGN, dict(x=A + 1)), (HP_EALIGN, dict(z=A + 1)), (HP_EALIGN, dict(w_pre=A + 1)), (HP_EALIGN, dict(rstd=A + 2)),
    (HP_OK, dict(rows=0)), (HP_OK, dict(rows=0, x=None, y=None, w_post=None, gate=None))])
def test_norm_refuses(code, kw):
    assert ops._lib().hp_gated_norm(C.byref(ops.hp_norm_args_t(**{**NORM, **kw})), None) == code


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(dh=None, dz=None)), (HP_EINVAL, dict(workspace=None)), (HP_EINVAL, dict(workspace_bytes=16)), (HP_EALIGN, dict(workspace=A + 8)),
    (HP_EALIGN, dict(dx=A + 1)), (HP_EALIGN, dict(dw_pre=A + 1)), (HP_EINVAL, dict(of=dict(rstd=None))), (HP_EINVAL, dict(of=dict(w_pre=None))),
    (HP_EINVAL, dict(of=dict(w_post=None))), (HP_EINVAL, dict(of=dict(gate=None))), (HP_EINVAL, dict(of=dict(y=None, w_post=None, gate=None))),
    (HP_OK, dict(of=dict(rows=0), dw_post=None, dgate=None, dw_pre=None)), (HP_OK, dict(dx=None, dy=None, dw_post=None, dgate=None, dw_pre=None))])
def test_norm_backward_refuses(code, kw):
    f = ops.hp_norm_args_t(**{**NORM, **kw.pop("of", {})})
    g = ops.hp_norm_grads_t(**{**dict(dh=A, dz=A, dh_stride=64, dz_stride=64, dx=A, dy=A, dx_stride=64, dy_stride=64, dw_post=A, dgate=A, dw_pre=A,
                                      workspace=A, workspace_bytes=1 << 30), **kw})
    L = ops._lib()
    assert L.hp_gated_norm_backward(C.byref(f), C.byref(g), None) == code
    assert L.hp_gated_norm_backward(C.byref(f), None, None) == HP_EINVAL and L.hp_gated_norm_backward(None, C.byref(g), None) == HP_EINVAL


def test_norm_workspace():
    for bad in ((-1, 64), (4, 0), (4, 32769)):
        with pytest.raises(HpError):
            hp.hp_gated_norm_workspace(*bad)
    sizes = [hp.hp_gated_norm_workspace(n, 4096) for n in (0, 1, 8, 100, 10 ** 9)]
    assert sizes == sorted(sizes) and 0 < sizes[-1] < 1 << 28
    assert all(hp.hp_gated_norm_workspace(5, h) >= 5 * 2 * h * 4 for h in range(1, 32769, 97))


# ---- cross attention ------------------------------------------------------------------------------------------------

def attend_args(**kw):
    d = dict(dtype=0, heads_q=8, heads_k=2, dim=64, rows=4, keys=6, scale=0.125, q=heads(), k=heads(), v=heads(), out=heads(), ranges=A, lse=A,
             workspace=A, workspace_bytes=1 << 40, dout=heads(), dq=heads(), dk=heads(), dv=heads())
    return ops.hp_attend_args_t(**{**d, **kw})


BOTH = [
    (HP_EINVAL, dict(dtype=7)), (HP_EINVAL, dict(dim=0)), (HP_EINVAL, dict(dim=257)), (HP_EINVAL, dict(heads_q=0)), (HP_EINVAL, dict(heads_k=0)),
    (HP_ELAYOUT, dict(heads_q=7)), (HP_ELAYOUT, dict(heads_q=16386)), (HP_EINVAL, dict(rows=-1)), (HP_EINVAL, dict(keys=-1)),
    (HP_ELAYOUT, dict(rows=(1 << 28) + 1)), (HP_ELAYOUT, dict(keys=(1 << 31) - 1)), (HP_EINVAL, dict(scale=0.0)), (HP_EINVAL, dict(scale=-1.0)),
    (HP_EINVAL, dict(scale=float("nan"))), (HP_EINVAL, dict(scale=float("inf"))), (HP_EINVAL, dict(q=heads(None))), (HP_EINVAL, dict(k=heads(None))),
    (HP_EINVAL, dict(v=heads(None))), (HP_EINVAL, dict(out=heads(None))), (HP_EALIGN, dict(q=heads(A + 1))), (HP_EALIGN, dict(v=heads(A + 1))),
    (HP_EALIGN, dict(ranges=A + 2)), (HP_EALIGN, dict(lse=A + 1)), (HP_EALIGN, dict(workspace=A + 4))]


@pytest.mark.parametrize("call", ["hp_cross_attend", "hp_cross_attend_step", "hp_cross_attend_backward"])
@pytest.mark.parametrize("code,kw", BOTH)
def test_attend_refuses(call, code, kw):
    assert getattr(ops._lib(), call)(C.byref(attend_args(**kw)), None) == code
    assert getattr(ops._lib(), call)(None, None) == HP_EINVAL


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(lse=None)), (HP_EINVAL, dict(dout=heads(None))), (HP_EINVAL, dict(dq=heads(None))), (HP_EINVAL, dict(dk=heads(None))),
    (HP_EINVAL, dict(dv=heads(None))), (HP_EALIGN, dict(dk=heads(A + 1))), (HP_EINVAL, dict(workspace=None)), (HP_EINVAL, dict(workspace_bytes=64)),
    (HP_OK, dict(rows=0, keys=0)), (HP_OK, dict(rows=0, keys=0, q=heads(None), k=heads(None), dv=heads(None), lse=None))])
def test_attend_backward_refuses(code, kw):
    assert ops._lib().hp_cross_attend_backward(C.byref(attend_args(**kw)), None) == code


def test_attend_without_rows_does_nothing_and_parts_need_scratch_memory():
    L = ops._lib()
    for call in (L.hp_cross_attend, L.hp_cross_attend_step):
        assert call(C.byref(attend_args(rows=0, q=heads(None), out=heads(None), workspace=None)), None) == HP_OK
        assert call(C.byref(attend_args(rows=1, keys=100000, workspace=None)), None) == HP_EINVAL
        assert call(C.byref(attend_args(rows=1, keys=100000, workspace_bytes=4)), None) == HP_EINVAL
    assert L.hp_cross_attend_step(C.byref(attend_args(rows=(1 << 23) + 1)), None) == HP_ELAYOUT


def test_attend_workspace():
    size = lambda call=0, **kw: ops._lib().hp_cross_attend_workspace(C.byref(attend_args(**kw)), call)  # noqa: E731
    assert size(3) == HP_EINVAL and size(-1) == HP_EINVAL and size(dim=300) == HP_EINVAL and size(heads_q=7) == HP_ELAYOUT
    assert size(0, rows=100000, keys=4000) == 0                       # rows enough: no parts
    assert size(0, rows=16, keys=40000) > 0 and size(1, rows=1, keys=576) > 0 and size(2) > 0
    assert max(size(c, rows=16, keys=40000) for c in range(3)) < 1 << 28


# ---- image ranges -----------------------------------------------------------------------------------------------------

def plain_ranges(tm, rule):
    out = np.zeros((tm.batch, tm.seq, 2), np.int64)
    first = np.concatenate([[0], np.cumsum(tm.img_len)])
    for b in range(tm.batch):
        own = [k for k in range(tm.n_images) if tm.img_sample[k] == b]
        base = first[own[0]] if own else first[sum(int(s) < b for s in tm.img_sample)]
        for p in range(tm.seq):
            see = [k for k in own if rule == "sample" or tm.img_start[k] + tm.img_len[k] <= p]
            see = see[-1:] if rule == "latest" else see
            out[b, p] = (first[see[0]], first[see[-1] + 1]) if see else (base, base)
    return out.reshape(-1, 2)


@pytest.mark.parametrize("rule", ["sample", "previous", "latest"])
def test_image_ranges(rule):
    maps = [wl.TokenMap(3, 20, 8, [0, 0, 0, 2], [0, 4, 13, 5], [4, 2, 7, 15]), wl.TokenMap(2, 5, 8, [], [], []),
            wl.TokenMap(1, 7, 8, [0], [0], [7])] + wl.tiny().maps
    for tm in maps:
        got = hp.hp_image_ranges(tm, rule)
        assert got.dtype == np.int32 and np.array_equal(got, plain_ranges(tm, rule))


def test_image_ranges_refuses():
    swapped = wl.TokenMap(1, 20, 8, [0, 0], [10, 0], [4, 4])
    assert hp.hp_image_ranges(swapped, "sample").tolist() == [[0, 8]] * 20
    with pytest.raises(ValueError):
        hp.hp_image_ranges(swapped, "next")
    for tm, rule in ((swapped, "previous"), (swapped, "latest"), (wl.TokenMap(1, 20, 8, [1], [0], [4]), "sample"),
                     (wl.TokenMap(2, 20, 8, [1, 0], [0, 0], [4, 4]), "sample"), (wl.TokenMap(1, 20, 8, [0], [18], [4]), "sample"),
                     (wl.TokenMap(1, 20, 8, [0], [3], [0]), "sample"), (wl.TokenMap(1, 20, 8, [0, 0], [3, 5], [4, 4]), "latest")):
        with pytest.raises(HpError) as e:
            hp.hp_image_ranges(tm, rule)
        assert e.value.code == HP_EMAP
    t, keep = ops._token_map(swapped)
    out = (C.c_int32 * 40)()
    assert ops._lib().hp_image_ranges(None, 0, out) == HP_EINVAL and ops._lib().hp_image_ranges(C.byref(t), 0, None) == HP_EINVAL
    assert ops._lib().hp_image_ranges(C.byref(t), 3, out) == HP_EINVAL


# ---- the binding's own checks -------------------------------------------------------------------------------------------

def test_the_binding_refuses_host_tensors():
    x = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    for call in (lambda: hp.hp_rotary([x], [x], torch.zeros(4, 4, 2), torch.zeros(4, dtype=torch.int32)),
                 lambda: hp.hp_rotary_table(torch.zeros(4, 4, 2)), lambda: hp.hp_gated_norm(x[:, 0], None, x[:, 0], None),
                 lambda: hp.hp_cross_attend(x, x, x, None, x), lambda: hp.hp_cross_attend_step(x, x, x, None, x)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="scaling"):
        hp.hp_rotary_table(x, scaling=hp.RotaryScaling("other"))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        hp.hp_cross_attend_workspace(x.half(), x.half())
