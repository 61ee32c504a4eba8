"""The host side of states and weights in 4 bits: what the calls refuse (before any HIP call, so without a GPU), scratch
sizes, the header against the binding, and how the attention's units share out tiles (csrc/hp_share.hpp, the kernels' own code)."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import packed_plain as plain
import paper_2605_27678_amd as hp
from paper_2605_27678_amd import packed as pk
from paper_2605_27678_amd.binding import HP_EALIGN, HP_EINVAL, HP_ELAYOUT, HP_OK
from paper_2605_27678_amd.operators import hp_heads_t

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                       # an address that no refused call looks at
TOO_FAR = (1 << 24) + 16


def heads(p=A, row=64, head=8):
    return hp_heads_t(p, row, head)


def packed(codes=A, scales=A, row=64, head=32, s_row=8, s_head=4):
    return pk.hp_packed_t(codes, scales, row, head, s_row, s_head)


def test_the_header_declares_what_the_binding_has():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hp_packed.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(hp_\w+)\s*\(", text)) == set(pk.EXPORTS)
    for name in pk.EXPORTS:
        assert getattr(pk._lib(), name) and name in hp.__all__
    assert "Packed" in hp.__all__ and f"HP_PACKED_GROUP   {pk.GROUP}" in text and f"HP_PACK_MAX_TENSORS {pk.MAX_TENSORS}" in text


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++11")])
def test_the_header_is_plain_c_and_its_structs_are_the_bindings(compiler, std, tmp_path):
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    names = ["hp_packed_t", "hp_pack_args_t", "hp_packed_attend_args_t", "hp_packed_linear_args_t"]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hp_packed.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", sizeof({n}));\n' for n in names) +
                   "".join(f'  printf("%zu\\n", offsetof({n}, {f}));\n' for n in names for f, *_ in getattr(pk, n)._fields_) +
                   "  return 0; }\n")
    exe = tmp_path / "t"
    subprocess.run([compiler, std, "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe)], check=True, capture_output=True, timeout=120)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, timeout=30).stdout.split()]
    structs = [getattr(pk, n) for n in names]
    assert got == [C.sizeof(s) for s in structs] + [getattr(s, f).offset for s in structs for f, *_ in s._fields_]


# ---- packing ---------------------------------------------------------------------------------------------------------

def pack_args(**kw):
    a = pk.hp_pack_args_t(dtype=0, n_tensors=2, dim=64, rows=4)
    for t in range(2):
        a.heads[t], a.x[t], a.packed[t] = 3, heads(), packed()
    for n, v in kw.items():
        if "_at_" in n:
            getattr(a, n.split("_at_")[0])[int(n[-1])] = v
        else:
            setattr(a, n, v)
    return a


BAD_PACKED = [(HP_EINVAL, packed(codes=None)), (HP_EINVAL, packed(scales=None)), (HP_EALIGN, packed(codes=A + 8)), (HP_EALIGN, packed(scales=A + 2)),
              (HP_EALIGN, packed(row=72)), (HP_EALIGN, packed(s_row=7)), (HP_EALIGN, packed(head=8)), (HP_EALIGN, packed(s_head=3))]


@pytest.mark.parametrize("call", ["hp_pack", "hp_unpack"])
@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(dtype=2)), (HP_EINVAL, dict(dtype=-1)), (HP_EINVAL, dict(n_tensors=0)), (HP_EINVAL, dict(n_tensors=5)), (HP_EINVAL, dict(rows=-1)),
    (HP_EINVAL, dict(dim=0)), (HP_EINVAL, dict(dim=65537)), (HP_EINVAL, dict(heads_at_1=-1)), (HP_EINVAL, dict(heads_at_0=65537)),
    (HP_EINVAL, dict(x_at_1=heads(None))), (HP_EALIGN, dict(x_at_0=heads(A + 1))), (HP_EALIGN, dict(dtype=1, x_at_0=heads(A + 2))),
    (HP_ELAYOUT, dict(dim=65536, heads_at_0=2048)),
    *((code, dict(packed_at_1=t)) for code, t in BAD_PACKED),
    (HP_OK, dict(rows=0)), (HP_OK, dict(heads_at_0=0, heads_at_1=0)), (HP_OK, dict(rows=0, x_at_0=heads(None), packed_at_0=packed(None, None)))])
def test_pack_refuses(call, code, kw):
    assert getattr(pk._lib(), call)(C.byref(pack_args(**kw)), None) == code


# ---- attention -------------------------------------------------------------------------------------------------------

def attend_args(**kw):
    d = dict(dtype=0, heads_q=8, heads_k=2, dim=64, rows=4, keys=6, scale=0.125, q=heads(), out=heads(), k=packed(), v=packed(), ranges=A, lse=A,
             workspace=A, workspace_bytes=1 << 60)
    return pk.hp_packed_attend_args_t(**{**d, **kw})


SIZES = [(HP_EINVAL, dict(dtype=2)), (HP_EINVAL, dict(dim=0)), (HP_EINVAL, dict(dim=257)), (HP_EINVAL, dict(heads_k=0)), (HP_EINVAL, dict(heads_q=0)),
         (HP_EINVAL, dict(rows=-1)), (HP_EINVAL, dict(keys=-1)), (HP_ELAYOUT, dict(heads_q=9)), (HP_ELAYOUT, dict(heads_q=16386)),
         (HP_ELAYOUT, dict(rows=(1 << 23) + 1)), (HP_ELAYOUT, dict(heads_q=16384, heads_k=2, rows=131072)), (HP_ELAYOUT, dict(keys=(1 << 31) - 1024))]


@pytest.mark.parametrize("code,kw", SIZES + [
    (HP_EINVAL, dict(scale=0.0)), (HP_EINVAL, dict(scale=-1.0)), (HP_EINVAL, dict(scale=float("nan"))), (HP_EINVAL, dict(scale=float("inf"))),
    (HP_EINVAL, dict(scale=3e38)), (HP_EINVAL, dict(q=heads(None))), (HP_EINVAL, dict(out=heads(None))), (HP_EALIGN, dict(q=heads(A + 1))),
    (HP_EALIGN, dict(dtype=1, out=heads(A + 2))), (HP_EALIGN, dict(ranges=A + 2)), (HP_EALIGN, dict(lse=A + 2)), (HP_EALIGN, dict(workspace=A + 8)),
    (HP_EINVAL, dict(workspace=None)), (HP_EINVAL, dict(workspace_bytes=15)),
    *((code, {which: t}) for which in "kv" for code, t in BAD_PACKED),
    (HP_ELAYOUT, dict(k=packed(row=TOO_FAR))), (HP_ELAYOUT, dict(v=packed(s_row=TOO_FAR))), (HP_ELAYOUT, dict(v=packed(row=-64))),
    (HP_ELAYOUT, dict(k=packed(s_row=-8))),
    (HP_OK, dict(rows=0, q=heads(None), out=heads(None), workspace=None)), (HP_OK, dict(rows=0, keys=0, k=packed(None, None))),
    # strides that no address goes by
    (HP_OK, dict(rows=0, keys=1, k=packed(row=-8, s_row=1))), (HP_OK, dict(rows=0, heads_q=4, heads_k=1, k=packed(head=7, s_head=1)))])
def test_attend_refuses(code, kw):
    assert pk._lib().hp_packed_attend_step(C.byref(attend_args(**kw)), None) == code


@pytest.mark.parametrize("code,kw", SIZES)
def test_the_scratch_memory_is_refused_where_the_call_is(code, kw):
    assert pk._lib().hp_packed_attend_workspace(C.byref(attend_args(**kw))) == code


def test_attend_workspace():
    size = lambda **kw: pk._lib().hp_packed_attend_workspace(C.byref(attend_args(**kw)))  # noqa: E731
    assert size(rows=0) == 0 and size(rows=100000) == 0              # nothing is shared out
    for kw in (dict(), dict(keys=0), dict(rows=1, keys=1 << 30), dict(rows=512, keys=100000, dim=256), dict(heads_q=16384, heads_k=16384), dict(heads_q=4080, heads_k=2)):
        n = size(**kw)
        assert n > 0 and n % 16 == 0
        need = dict(attend=C.byref(attend_args(workspace_bytes=n - 1, **kw)))
        assert pk._lib().hp_packed_attend_step(need["attend"], None) == HP_EINVAL
    # few hundred megabytes at most, whatever the sizes: of every state head two partial results a unit
    assert size(rows=512, keys=1 << 21, heads_q=16384, heads_k=1024, dim=256) < 1 << 29
    L = pk._lib()
    assert L.hp_packed_attend_workspace(None) == HP_EINVAL and L.hp_packed_attend_step(None, None) == HP_EINVAL
    assert L.hp_pack(None, None) == L.hp_unpack(None, None) == L.hp_packed_linear(None, None) == HP_EINVAL


def test_several_rows_of_few_states_are_not_one_workgroups():
    """A workgroup goes through its rows one behind the other.  The scratch memory says how many units share them: two places of
    partial results each."""
    size = lambda **kw: pk._lib().hp_packed_attend_workspace(C.byref(attend_args(**kw)))  # noqa: E731
    whole = lambda n: (n + 15) // 16 * 16  # noqa: E731
    for heads_q, heads_k, dim in ((32, 8, 128), (1, 1, 64), (16, 2, 256), (16, 16, 72)):
        for dtype in (0, 1):
            of = lambda units, rows: whole(4 * 2 * units * heads_q * dim) + whole(4 * 2 * units * heads_q) + whole(8 * rows)  # noqa: E731
            sizes = dict(dtype=dtype, heads_q=heads_q, heads_k=heads_k, dim=dim)
            for rows, keys in ((2, 0), (2, 120), (2, 447), (3, 319), (5, 190), (8, 127), (15, 61), (16, 63), (16, 0)):
                assert size(rows=rows, keys=keys, **sizes) >= of(rows, rows)
            assert size(rows=1, keys=800, **sizes) == of(1, 1)         # a single one's are


# ---- linear ----------------------------------------------------------------------------------------------------------

def linear_args(**kw):
    d = dict(dtype=0, n_in=64, n_out=6, rows=4, x=A, x_stride=64, w=packed(), out=A, out_stride=6)
    return pk.hp_packed_linear_args_t(**{**d, **kw})


@pytest.mark.parametrize("code,kw", [
    (HP_EINVAL, dict(dtype=2)), (HP_EINVAL, dict(rows=-1)), (HP_EINVAL, dict(n_in=0)), (HP_EINVAL, dict(n_out=-1)), (HP_ELAYOUT, dict(n_in=65537)),
    (HP_ELAYOUT, dict(n_out=(1 << 24) + 1)), (HP_ELAYOUT, dict(rows=(1 << 20) + 1)), (HP_EINVAL, dict(x=None)), (HP_EINVAL, dict(out=None)),
    (HP_EALIGN, dict(x=A + 1)), (HP_EALIGN, dict(out=A + 1)), (HP_EALIGN, dict(dtype=1, x=A + 2)), (HP_EALIGN, dict(dtype=1, out=A + 2)),
    *((code, dict(w=t)) for code, t in BAD_PACKED[:6]), (HP_ELAYOUT, dict(w=packed(row=TOO_FAR))), (HP_ELAYOUT, dict(w=packed(s_row=-8))),
    (HP_OK, dict(rows=0, x=None, out=None)), (HP_OK, dict(n_out=0, out=None, w=packed(None, None))), (HP_OK, dict(rows=0, w=packed(head=7, s_head=1)))])
def test_linear_refuses(code, kw):
    assert pk._lib().hp_packed_linear(C.byref(linear_args(**kw)), None) == code


# ---- the binding's own checks ------------------------------------------------------------------------------------------

def test_the_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.bfloat16)
    room, matrix = hp.Packed.room(4, 2, 64, "cpu"), hp.Packed.room(4, None, 64, "cpu")
    for call in (lambda: hp.hp_pack([x], [room]), lambda: hp.hp_unpack([room], [x]), lambda: hp.hp_packed_attend_step(x, room, room, None, x),
                 lambda: hp.hp_packed_linear(w, matrix, w)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="as many packed"):
        hp.hp_pack([], [])
    with pytest.raises(ValueError, match="as many packed"):
        hp.hp_pack([x] * 5, [room] * 5)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        hp.hp_packed_attend_workspace(x.half(), room)


def test_room_for_packed_rows():
    for heads_k, dim in ((3, 64), (1, 72), (2, 1)):
        p = hp.Packed.room(5, heads_k, dim, "cpu")
        g = plain.groups(dim)
        assert p.codes.shape == (5, heads_k, 16 * g) and p.scales.shape == (5, heads_k, g, 2) and p.codes.stride(0) == 16 * g
        part = p.rows(2, 4)
        assert part.codes.shape[0] == part.scales.shape[0] == 2 and part.codes.data_ptr() == p.codes.data_ptr() + 32 * g
    p = hp.Packed.room(5, None, 72, "cpu")
    assert p.codes.shape == (5, 48) and p.scales.shape == (5, 3, 2)


def test_the_plain_form_reads_back_what_it_wrote():
    codes = torch.randint(0, 16, (3, 2, 32), generator=torch.Generator().manual_seed(0))
    assert torch.equal(plain.from_bytes(plain.to_bytes(codes)), codes)
    one = torch.zeros(1, 1, 32, dtype=torch.int64)
    one[0, 0, 8 * 2 + 2 * 1 + 1] = 5                                 # word 2, bits 20 to 23
    assert plain.to_bytes(one)[0].tolist() == [0] * 10 + [5 << 4] + [0] * 5


# ---- shares ------------------------------------------------------------------------------------------------------------

def test_units_share_out_all_tiles_evenly(tmp_path):
    exe, csrc = tmp_path / "walk_share", os.path.join(ROOT, "paper_2605_27678_amd", "csrc")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-Wall", "-I", csrc,
                        os.path.join(ROOT, "tests", "walk_share.cpp"), "-o", str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
