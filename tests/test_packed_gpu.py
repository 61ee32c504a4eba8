"""States and weights held in 4 bits on the GPU against their definitions in 64 bits (packed_plain.py)."""
import pytest
import torch

import packed_plain as plain
import paper_2605_27678_amd as hp
from operators_plain import BF16, F32, check, unit

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def rand(seed, *shape, dtype=BF16, scale=1.0, around=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (around + scale * torch.randn(shape, generator=g, device=DEV)).to(dtype)


def bytes_of(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def packed_of(x, layout="head"):
    """x packed by the library, into rows of heads that lie head by head, row by row, or with room between them."""
    if x.dim() == 2:
        p = hp.Packed.room(x.shape[0], None, x.shape[1], DEV)
    elif layout == "head":
        p = hp.Packed.room(*x.shape, DEV)
    else:
        g, more = plain.groups(x.shape[2]), (1 if layout == "wide" else 0)
        codes = torch.zeros(x.shape[0], x.shape[1] + more, 16 * (g + more), dtype=torch.uint8, device=DEV)
        scales = torch.zeros(x.shape[0], x.shape[1] + more, g + more, 2, dtype=BF16, device=DEV)
        p = hp.Packed(codes[:, :x.shape[1], :16 * g], scales[:, :x.shape[1], :g])
    hp.hp_pack([x], [p])
    return p


# ---- packing and reading back ------------------------------------------------------------------------------------

def same_packed(x, p):
    codes, step, low = plain.pack(x)
    assert torch.equal(p.codes, plain.to_bytes(codes))
    assert torch.equal(torch.nan_to_num(p.scales.double(), 1e30), torch.nan_to_num(torch.stack([step, low], -1), 1e30))
    return codes, step, low


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,heads,dim", [(1, 1, 1), (5, 3, 7), (4, 2, 31), (3, 5, 32), (17, 8, 128), (33, 2, 72), (9, 3, 100), (300, 8, 128),
                                            (2, 16, 256), (130, 1, 80), (7, 70, 64), (1, 2, 4099), (3, None, 2305), (70, None, 64)])
def test_pack_and_back(dtype, rows, heads, dim):
    shape = (rows, dim) if heads is None else (rows, heads, dim)
    x = rand(rows + dim, *shape, dtype=dtype, around=0.3)
    for layout in ("head", "row", "wide"):
        p = packed_of(x, layout)
        same_packed(x, p)
        back = torch.full_like(x, 9.0)
        hp.hp_unpack([p], [back])
        exact = plain.values(p, dim)
        check("values", back, exact, unit(dtype) * exact.abs() + 2.0 ** -23 * (exact.abs() + x.double().abs()))
        step = p.scales[..., 0].double().repeat_interleave(32, -1)[..., :dim]
        assert bool(((exact - x.double()).abs() <= step / 2).all())


def test_keys_and_values_of_other_heads_in_one_call_and_strided():
    whole = rand(1, 40, 3, 5, 41)                                        # q, k, v of one projection; odd strides
    k, v, x = whole[:, 1, :, :40], whole[:, 2, :2, 1:41], rand(2, 40, 7, 40)
    ps = [hp.Packed.room(64, t.shape[1], 40, DEV) for t in (k, v, x)]
    for p in ps:
        p.codes.fill_(0x5a)
        p.scales.fill_(3.0)
    hp.hp_pack([k, v, x], [p.rows(11, 51) for p in ps])
    back = torch.zeros(40, 14, 45, dtype=BF16, device=DEV)
    outs = [back[:, :5, 1:41], back[:, 5:7, 2:42], back[:, 7:, :40]]
    hp.hp_unpack([p.rows(11, 51) for p in ps], outs)
    for t, p, o in zip((k, v, x), ps, outs):
        same_packed(t, p.rows(11, 51))
        for edge in (p.rows(0, 11), p.rows(51, 64)):
            assert bool((edge.codes == 0x5a).all()) and bool((edge.scales == 3.0).all())
        exact = plain.values(p.rows(11, 51), 40)
        check("values", o, exact, unit(BF16) * exact.abs() + 2.0 ** -22 * exact.abs().amax())
    assert not bool(back[:, :5, 0].any()) and not bool(back[:, 7:, 40:].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_at_the_borders_of_levels(dtype):
    """Levels 0 .. 15 and whole numbers of 64ths between them: ties go to the lower; with values whose difference from the
    least is rounded in binary32; of one sign; all alike; tiny, huge and spread over the whole range."""
    n = torch.arange(961, device=DEV) / 64
    rows = [torch.cat([torch.tensor([0.0, 15.0], device=DEV), c]) for c in n.split(30)]
    x = torch.zeros(len(rows), 32, device=DEV)
    for i, r in enumerate(rows):
        x[i, :len(r)] = r
    tiny = x.clone()
    tiny[:, 2] = -2.0 ** -30
    wide = rand(3, 40, 32, dtype=F32) * torch.exp2(torch.randint(-40, 3, (40, 32), device=DEV, generator=torch.Generator(device=DEV).manual_seed(4)).float())
    many = torch.cat([x, tiny, x + 1.0, -x, x * 2.0 ** -120, x * 2.0 ** -128, x * 2.0 ** 123, x - 7.5, wide, 2.0 ** 120 * wide,
                      torch.full((3, 32), 0.1, device=DEV), torch.zeros(2, 32, device=DEV), (x - 7.5) * 2.0 ** 124]).to(dtype)
    same_packed(many, packed_of(many))


def test_values_that_are_not_finite():
    x = rand(5, 12, 2, 72, dtype=F32)
    for i, bad in enumerate((float("nan"), float("inf"), -float("inf"), -3.4e38, 3.4e38)):
        x[i, 0, 40 + i] = bad
        x[i, 1, 71] = bad
    p = packed_of(x)
    same_packed(x, p)
    assert bool(torch.isnan(p.scales[:4, 0, 1]).all()) and not bool(torch.isnan(p.scales[:, 0, 0]).any()) and not bool(torch.isnan(p.scales[4:]).any())
    back = torch.empty_like(x)
    hp.hp_unpack([p], [back])
    assert bool(torch.isnan(back[:4, 0, 32:64]).all()) and bool(torch.isfinite(back[5:]).all()) and bool(torch.isfinite(back[:, :, :32]).all())


# ---- attention ------------------------------------------------------------------------------------------------------

def attend_run(q, k, v, ranges, scale=None, lse=True):
    out = torch.full_like(q, 7.0)
    stats = torch.full(q.shape[:2], 7.0, dtype=F32, device=DEV) if lse else None
    hp.hp_packed_attend_step(q, k, v, ranges, out, lse=stats, scale=scale, workspace=bytes_of(hp.hp_packed_attend_workspace(q, k)))
    return out, stats


def ranges_of(*pairs):
    return torch.tensor(pairs, dtype=torch.int32, device=DEV)


def attend_check(q, k, v, ranges, scale=None):
    out, lse = attend_run(q, k, v, ranges, scale)
    want = plain.attend(q, k, v, ranges, q.shape[2] ** -0.5 if scale is None else scale)
    check("out", out, *want["out"])
    check("lse", lse, *want["lse"])
    return out, lse


LENGTHS = (0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 255, 256, 257, 300)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads_q,heads_k,dim", [(1, 1, 1), (2, 1, 8), (3, 3, 31), (8, 2, 33), (8, 2, 64), (5, 5, 72), (6, 2, 80), (16, 1, 96), (17, 1, 100),
                                                 (8, 1, 128), (40, 2, 128), (4, 2, 130), (3, 1, 200), (16, 2, 256)])
def test_attend_step(dtype, heads_q, heads_k, dim):
    starts = [3]
    for n in LENGTHS:
        starts.append(starts[-1] + n + 1)
    keys = starts[-1] + 2
    q = rand(1, len(LENGTHS) + 4, heads_q, dim, dtype=dtype)
    k, v = rand(2, keys, heads_k, dim, dtype=dtype, around=0.5), rand(3, keys, heads_k, dim, dtype=dtype, around=-0.25)
    ranges = ranges_of(*((a, a + n) for a, n in zip(starts, LENGTHS)), (-5, 4), (keys - 3, keys + 9), (9, 2), (keys, keys + 1))
    for layout in ("head", "row", "wide"):
        out, lse = attend_check(q, packed_of(k, layout), packed_of(v, layout), ranges)
        assert not bool(out[0].any()) and bool((lse[0] == float("-inf")).all()) and not bool(out[-2:].any())
    attend_check(q[:2], packed_of(k), packed_of(v), None, 0.3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,keys,heads_q,heads_k,dim", [(1, 5000, 8, 2, 128), (2, 20011, 2, 1, 64), (3, 3000, 4, 4, 256), (1, 70000, 1, 1, 32), (40, 2500, 8, 8, 80)])
def test_attend_step_over_parts(dtype, rows, keys, heads_q, heads_k, dim):
    q, k, v = rand(1, rows, heads_q, dim, dtype=dtype), packed_of(rand(2, keys, heads_k, dim, dtype=dtype)), packed_of(rand(3, keys, heads_k, dim, dtype=dtype))
    assert hp.hp_packed_attend_workspace(q, k) > 0
    attend_check(q, k, v, None)
    n = torch.arange(rows, device=DEV, dtype=torch.int32) * 7
    attend_check(q, k, v, torch.stack([n, n + keys // 3], 1).contiguous())


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_states_that_are_not_seen_have_no_influence(dim):
    rows, keys = 6, 1500
    q, k, v = rand(1, rows, 8, dim), packed_of(rand(2, keys, 2, dim)), packed_of(rand(3, keys, 2, dim))
    ranges = ranges_of((0, 100), (200, 265), (300, 301), (301, 301), (700, 1400), (1499, 1500))
    want = attend_run(q, k, v, ranges)
    seen = torch.zeros(keys, dtype=torch.bool, device=DEV)
    for a, b in ranges.tolist():
        seen[a:b] = True
    for t in (k, v):
        t.scales[~seen] = float("nan")
        t.codes[~seen] = 0xff
    got = attend_run(q, k, v, ranges)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_states_that_are_seen_and_not_finite():
    q, k, v = rand(1, 4, 4, 128), packed_of(rand(2, 400, 2, 128)), packed_of(rand(3, 400, 2, 128))
    ranges = ranges_of((0, 100), (100, 200), (200, 300), (300, 400))
    want, _ = attend_run(q, k, v, ranges)
    v.scales[150, 0, 2] = float("nan")                                   # one group of one state head
    k.scales[250, 1, 0] = float("nan")
    got, lse = attend_run(q, k, v, ranges)
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[1, :2, 64:96] = True
    nan[2, 2:] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    assert bool(torch.isnan(lse[2, 2:]).all()) and int(torch.isnan(lse).sum()) == 2


def test_large_scores_and_far_maxima():
    """Scores that grow along the range, so that the running maximum is raised again and again, and such that all but one
    weight vanish."""
    dim, keys = 64, 1000
    k = rand(1, keys, 1, dim, dtype=F32) * (1 + torch.arange(keys, device=DEV)[:, None, None] / 20)
    for dtype in (BF16, F32):
        q, v = rand(2, 2, 4, dim, dtype=dtype), packed_of(rand(3, keys, 1, dim, dtype=dtype))
        attend_check(q, packed_of(k.to(dtype)), v, None, 1.0)
        attend_check(q, packed_of(k.flip(0).contiguous().to(dtype)), v, None, 1.0)


def test_outputs_that_are_small_beside_the_values():
    """Means of 8000 values around zero.  A wave of a row's four adds up 2000 of them in 32 tiles, in six products each at most; every
    addition rounds by half a step of what it has then, and 200 such roundings come to six times the root of their number at most.
    (What cancels, steps against lows, has 20 times their size and may not add up by itself.)"""
    rows, keys, dim = 600, 8000, 64
    k, v = packed_of(rand(2, keys, 1, dim, dtype=F32)), packed_of(rand(3, keys, 1, dim, dtype=F32))
    q = rand(4, 1, 1, dim, dtype=F32).expand(rows, 1, dim)
    out, _ = attend_run(q, k, v, None)
    p = torch.softmax(plain.values(k, dim)[:, 0] @ q[0, 0].double() * dim ** -0.5, 0)
    terms = p[:, None] * plain.values(v, dim)[:, 0]
    most = sum(terms[64 * w:].unfold(0, 64, 256).sum(-1).cumsum(0).abs().amax(0) for w in range(4))
    # and the weights themselves: their exponents' roundings, of unlike signs too
    weights = 6 * (terms * terms).sum(0).sqrt() * 2.0 ** -20
    apart = (out.double()[:, 0] - terms.sum(0)).abs()
    assert float((apart - (6 * 200 ** 0.5 * 2.0 ** -24 * most + weights)).max()) <= 0


# ---- linear ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1), (1, 32, 16), (2, 33, 17), (3, 128, 64), (1, 4096, 300), (16, 512, 48), (17, 1000, 40), (32, 256, 130),
                                             (33, 777, 65), (64, 640, 96), (65, 2305, 33), (130, 96, 20), (5, 65536, 18), (4, 160, 5000)])
def test_linear(dtype, rows, n_in, n_out):
    x, w = rand(1, rows, n_in, dtype=dtype), rand(2, n_out, n_in, dtype=dtype, scale=n_in ** -0.5, around=0.1)
    p = packed_of(w)
    out = torch.full((rows, n_out), 7.0, dtype=dtype, device=DEV)
    hp.hp_packed_linear(x, p, out)
    check("out", out, *plain.linear(x, p))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_linear_of_strided_tensors(dtype):
    x = rand(1, 9, 3, 211, dtype=dtype)[:, 1, 1:210]
    w = rand(2, 70, 209, dtype=dtype)
    codes, scales = torch.zeros(70, 16 * 9, dtype=torch.uint8, device=DEV), torch.full((70, 9, 2), float("nan"), dtype=BF16, device=DEV)
    p = hp.Packed(codes[:, :16 * 7], scales[:, :7])
    hp.hp_pack([w], [p])
    out = torch.full((9, 100), 7.0, dtype=dtype, device=DEV)
    hp.hp_packed_linear(x, p.rows(5, 65), out[:, 3:63])
    check("out", out[:, 3:63], *plain.linear(x, p.rows(5, 65)))
    assert bool((out[:, :3] == 7.0).all()) and bool((out[:, 63:] == 7.0).all())


def test_linear_rows_that_are_not_finite_stay_by_themselves():
    x, p = rand(1, 20, 300), packed_of(rand(2, 50, 300))
    clean, out = torch.empty(20, 50, dtype=BF16, device=DEV), torch.empty(20, 50, dtype=BF16, device=DEV)
    hp.hp_packed_linear(x, p, clean)
    x[3, 299], x[18, 0] = float("inf"), float("nan")
    hp.hp_packed_linear(x, p, out)
    fine = [i for i in range(20) if i not in (3, 18)]
    assert torch.equal(out[fine], clean[fine]) and bool(torch.isnan(out[[3, 18]]).all())
