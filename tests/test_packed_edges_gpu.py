"""States and weights held in 4 bits where calls are cut differently, lie far apart, are captured, or follow one another."""
import pytest
import torch

import packed_plain as plain
import paper_2605_27678_amd as hp
from operators_plain import BF16, F32, check, sums, unit
from paper_2605_27678_amd import operators as ops
from test_packed_gpu import DEV, attend_check, attend_run, bytes_of, packed_of, rand, ranges_of

pytestmark = pytest.mark.gpu


# ---- linear: every tile that a call can choose -------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 1056, 300), (4, 160, 66000), (2, 1056, 8200), (4, 1024, 12300), (2, 1040, 16400), (16, 1056, 4100), (9, 1032, 8200),
                                             (16, 1024, 12300), (16, 1024, 16400), (17, 1056, 4100), (32, 1024, 9000), (33, 512, 4090), (40, 1024, 9000), (64, 1056, 8210),
                                             (65, 512, 700), (130, 1024, 4100), (200, 96, 70)])
def test_linear_in_all_cuts(dtype, rows, n_in, n_out):
    x, w = rand(1, rows, n_in, dtype=dtype, around=0.25), packed_of(rand(2, n_out, n_in, dtype=BF16, scale=n_in ** -0.5))
    wide = torch.full((rows + 2, n_out + 3), 7.0, dtype=dtype, device=DEV)
    out = wide[1:rows + 1, 1:n_out + 1]
    want = plain.linear(x, w)
    hp.hp_packed_linear(x, w, out)
    check("out", out, *want)
    # rows that do not begin at whole pieces pass through registers
    apart = torch.empty(rows, n_in + 1, dtype=dtype, device=DEV)[:, 1:]
    apart.copy_(x)
    hp.hp_packed_linear(apart, w, out)
    check("out of odd rows", out, *want)
    out.fill_(7.0)
    assert bool((wide == 7.0).all())                                   # nothing beside the rows and columns


def test_linear_says_the_same_every_time():
    x, w = rand(1, 40, 4096), packed_of(rand(2, 5000, 4096))
    outs = [torch.empty(40, 5000, dtype=BF16, device=DEV) for _ in range(4)]
    for out in outs:
        hp.hp_packed_linear(x, w, out)
    assert all(torch.equal(out, outs[0]) for out in outs)


def test_one_row_of_any_stride_and_one_output():
    """Strides that no address goes by."""
    x = rand(1, 1, 512).as_strided((1, 512), (1 << 40, 1))
    p = packed_of(rand(2, 1, 512))
    w = hp.Packed(p.codes.as_strided(p.codes.shape, (16 << 40, 1)), p.scales.as_strided(p.scales.shape, (1 << 40, 2, 1)))
    out = torch.empty(1, 1, dtype=BF16, device=DEV)
    hp.hp_packed_linear(x, w, out)
    check("out", out, *plain.linear(x, p))
    k = packed_of(rand(3, 1, 1, 512 // 4))
    far = hp.Packed(k.codes.as_strided(k.codes.shape, (16 << 40, 16 << 40, 1)), k.scales.as_strided(k.scales.shape, (1 << 40, 1 << 40, 2, 1)))
    q = rand(4, 2, 3, 128)
    got, want = attend_run(q, far, far, ranges_of((0, 1), (-3, 5))), attend_run(q, k, k, None)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- attention: how rows are shared out --------------------------------------------------------------------------------

def ragged(seed, rows, keys, most):
    g = torch.Generator().manual_seed(seed)
    lo = torch.randint(-5, keys, (rows,), generator=g)
    n = torch.randint(0, most, (rows,), generator=g) * (torch.rand(rows, generator=g) < 0.9)
    return torch.stack([lo, lo + n], 1).to(torch.int32).to(DEV).contiguous()


@pytest.mark.parametrize("rows,heads_q,heads_k,dim,keys,most", [(63, 2, 1, 64, 700, 300), (64, 1, 1, 128, 900, 600), (65, 2, 2, 72, 700, 300), (511, 1, 1, 64, 3000, 200),
                                                                (512, 1, 1, 256, 900, 100), (513, 1, 1, 128, 2000, 300), (600, 2, 1, 96, 500, 100), (7, 40, 2, 128, 9000, 7000),
                                                                (3, 33, 1, 256, 3000, 2500), (5, 70, 70, 64, 700, 400), (2, 300, 300, 32, 300, 200)])
def test_ragged_rows_of_all_numbers(rows, heads_q, heads_k, dim, keys, most):
    q, k, v = rand(1, rows, heads_q, dim), packed_of(rand(2, keys, heads_k, dim)), packed_of(rand(3, keys, heads_k, dim, around=0.5))
    assert (hp.hp_packed_attend_workspace(q, k) > 0) == (rows <= 512)
    ranges = ragged(4, rows, keys, most)
    ranges[rows // 2] = torch.tensor([0, keys])
    attend_check(q, k, v, ranges)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_row_that_sees_much_among_many_that_see_little(dtype):
    rows, keys = 100, 30000
    q, k, v = rand(1, rows, 1, 128, dtype=dtype), packed_of(rand(2, keys, 1, 128)), packed_of(rand(3, keys, 1, 128))
    for at in (0, 57, rows - 1):
        ranges = ragged(4, rows, keys, 5)
        ranges[at] = torch.tensor([3, keys - 2])
        out, lse = attend_run(q, k, v, ranges)
        again = attend_run(q, k, v, ranges)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
        only = torch.arange(max(0, at - 3), min(rows, at + 4), device=DEV)
        want = plain.attend(q[only], k, v, ranges[only], 128 ** -0.5)
        check("out", out[only], *want["out"])
        check("lse", lse[only], *want["lse"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads_q,heads_k,dim", [(4, 2, 64), (12, 2, 72), (40, 2, 128), (2, 1, 160), (12, 2, 256)])
def test_a_seen_nan_stays_however_the_row_is_cut(dtype, heads_q, heads_k, dim):
    """Scores of neighbouring states one apart, so that all weights but those of the last hundred states are zero.  A state that is
    seen and NaN in a group of v leaves NaN in that group, wherever it lies: in the part of another unit than the greatest score,
    another wave's tile, or the same tile."""
    keys, group = 6000, heads_q // heads_k
    k, v = packed_of(torch.arange(keys, device=DEV, dtype=F32)[:, None, None].expand(keys, heads_k, dim).contiguous()), packed_of(rand(3, keys, heads_k, dim))
    one = torch.ones(1, heads_q, dim, dtype=dtype, device=DEV)
    groups = plain.groups(dim)
    for rows, n in ((1, keys), (5, keys), (520, 4000), (1, 500)):       # cut among units, five rows of them, a workgroup each, one workgroup
        q = one.expand(rows, heads_q, dim).contiguous()
        first = keys - n
        ranges = ranges_of((first, keys)).expand(rows, 2).contiguous()
        want = attend_run(q, k, v, ranges, 1.0 / dim)
        assert bool(torch.isfinite(want[0]).all())
        for at in (first, first + 70, first + n // 3, keys - 200, keys - 1):
            g, bad = at % groups, hp.Packed(v.codes, v.scales.clone())
            bad.scales[at, 0, g, at % 2] = float("nan")                  # step or low of a group of the first state head
            got = attend_run(q, k, bad, ranges, 1.0 / dim)
            nan = torch.zeros_like(got[0], dtype=torch.bool)
            nan[:, :group, 32 * g:32 * g + 32] = True
            assert torch.equal(torch.isnan(got[0]), nan), (rows, at - first)
            assert torch.equal(got[0][~nan], want[0][~nan]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads_q,heads_k,dim", [(8, 2, 64), (3, 3, 72), (17, 1, 128), (16, 2, 256)])
def test_a_few_rows_of_a_few_states(dtype, heads_q, heads_k, dim):
    for rows, keys in ((1, 1), (1, 63), (1, 900), (2, 1), (2, 447), (3, 319), (5, 190), (8, 127), (15, 61), (16, 63)):
        q, k, v = rand(1, rows, heads_q, dim, dtype=dtype), packed_of(rand(2, keys, heads_k, dim, dtype=dtype)), packed_of(rand(3, keys, heads_k, dim, dtype=dtype))
        attend_check(q, k, v, None)
        lo = torch.arange(rows) * keys // rows
        ranges = torch.stack([lo, (torch.arange(rows) + 1) * keys // rows], 1).to(torch.int32).to(DEV).contiguous()
        out, lse = attend_check(q, k, v, ranges)
        none = ranges[:, 0] == ranges[:, 1]
        assert not bool(out[none].any()) and bool((lse[none] == float("-inf")).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,dim", [(1030, 32), (600, 128), (260, 256)])
def test_several_rows_of_so_many_heads_that_each_has_one_unit(dtype, heads, dim):
    rows, keys = 9, 300
    q, k, v = rand(1, rows, heads, dim, dtype=dtype), packed_of(rand(2, keys, heads, dim)), packed_of(rand(3, keys, heads, dim))
    ranges = ranges_of((0, 300), (5, 5), (7, 8), (0, 64), (1, 66), (250, 400), (9, 2), (100, 229), (299, 300))
    out, lse = attend_run(q, k, v, ranges)
    for h in (slice(0, 3), slice(heads - 3, heads)):
        want = plain.attend(q[:, h], hp.Packed(k.codes[:, h], k.scales[:, h]), hp.Packed(v.codes[:, h], v.scales[:, h]), ranges, dim ** -0.5)
        check("out", out[:, h], *want["out"])
        check("lse", lse[:, h], *want["lse"])


def test_rows_that_all_see_nothing():
    for rows, keys in ((1, 50), (3, 5000), (200, 900), (600, 10), (4, 0)):
        q, k = rand(1, rows, 4, 64), packed_of(rand(2, keys, 2, 64))
        out, lse = attend_run(q, k, k, torch.zeros(rows, 2, dtype=torch.int32, device=DEV))
        assert not bool(out.any()) and bool((lse == float("-inf")).all())
    out, lse = attend_run(q, k, k, None)
    assert not bool(out.any()) and bool((lse == float("-inf")).all())


def test_what_the_scratch_memory_and_the_places_beside_the_output_hold():
    q, k, v = rand(1, 9, 6, 80), packed_of(rand(2, 6000, 2, 80)), packed_of(rand(3, 6000, 2, 80))
    want = attend_run(q, k, v, None)
    size = hp.hp_packed_attend_workspace(q, k)
    results = []
    for value in (0x00, 0xff, 0x7f):
        scratch = torch.full((size + 256,), value, dtype=torch.uint8, device=DEV)
        wide = torch.full((11, 8, 81), 7.0, dtype=BF16, device=DEV)
        out = wide[1:10, 1:7, :80]
        hp.hp_packed_attend_step(q, k, v, None, out, workspace=scratch[:size])
        assert torch.equal(out, want[0]) and bool((scratch[size:] == value).all())
        results.append(out.clone())
        out.fill_(7.0)
        assert bool((wide == 7.0).all())
    with pytest.raises(hp.HpError):
        hp.hp_packed_attend_step(q, k, v, None, out, workspace=scratch[:size - 1])
    with pytest.raises(hp.HpError):
        hp.hp_packed_attend_step(q, k, v, None, out)


def test_the_most_rows():
    """2^23 rows, which see two states at most."""
    rows, dim = 1 << 23, 8
    q = torch.empty(rows, 1, dim, dtype=BF16, device=DEV)
    q[:] = rand(1, 64, 1, dim).repeat(rows // 64, 1, 1)
    k, v = packed_of(rand(2, 66, 1, dim)), packed_of(rand(3, 66, 1, dim))
    lo = torch.arange(64, dtype=torch.int32, device=DEV)
    few = torch.stack([lo, lo + lo % 3], 1).contiguous()
    out, _ = attend_run(q, k, v, few.repeat(rows // 64, 1), lse=False)
    want, _ = attend_run(q[:64], k, v, few)
    assert torch.equal(out.view(-1, 64, 1, dim), want[None].expand(rows // 64, -1, -1, -1))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads_q,heads_k,dim", [(6, 2, 64), (12, 2, 96), (4, 4, 256)])
def test_queries_that_are_not_finite_stay_by_themselves(dtype, heads_q, heads_k, dim):
    q, k, v = rand(1, 5, heads_q, dim, dtype=dtype), packed_of(rand(2, 900, heads_k, dim)), packed_of(rand(3, 900, heads_k, dim))
    ranges = ranges_of((0, 900), (5, 300), (7, 7), (100, 200), (0, 64))
    want, _ = attend_run(q, k, v, ranges)
    q[0, 1, 3], q[1, heads_q - 1, dim - 1], q[2, 0, 0], q[3, 2, 1] = float("inf"), float("nan"), float("nan"), -float("inf")
    got, _ = attend_run(q, k, v, ranges)
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[0, 1] = nan[1, heads_q - 1] = nan[3, 2] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_and_small_values(dtype):
    q, k, v = rand(1, 4, 6, 96, dtype=dtype), rand(2, 500, 2, 96, dtype=dtype), rand(3, 500, 2, 96, dtype=dtype, around=0.5)
    x, w = rand(4, 5, 320, dtype=dtype), rand(5, 70, 320, dtype=dtype)
    for size in (2.0 ** 60, 2.0 ** -60):
        attend_check(q * size, packed_of(k / size), packed_of(v * size), None)
        out = torch.empty(5, 70, dtype=dtype, device=DEV)
        for a, b in ((x * size, w), (x, w * size), (x * size, w / size)):
            p = packed_of(b)
            hp.hp_packed_linear(a, p, out)
            check("out", out, *plain.linear(a, p))


@pytest.mark.parametrize("dtype,most", [(BF16, 118), (F32, 122)])
def test_the_largest_values_whose_sums_are_safe(dtype, most):
    """Activations and queries of one sign right below the sizes that the header names.  A group's sum of |x| is 2^(most + 5) at
    most; weights below 2^-4 leave 8 times what adds up over ten groups below 2^128."""
    g = torch.Generator(device=DEV).manual_seed(7)
    largest = 2.0 ** most * (1 - unit(dtype))
    for rows in (3, 16, 40):
        x = (largest * (1 - torch.rand(rows, 320, generator=g, device=DEV) / 64)).to(dtype)
        x[1], x[2, 7:] = largest, -largest
        for n_in, w in ((320, 2.0 ** -4 * (2 * torch.rand(50, 320, generator=g, device=DEV) - 1)), (317, torch.full((50, 317), 2.0 ** -20, device=DEV))):
            p, out = packed_of(w.to(dtype)), torch.empty(rows, 50, dtype=dtype, device=DEV)
            a = x[:, :n_in].contiguous()
            assert float(a.abs().max()) == largest
            hp.hp_packed_linear(a, p, out)
            check("out", out, *plain.linear(a, p))
    for heads_q, heads_k, dim in ((6, 2, 96), (5, 1, 256)):
        q, k, v = torch.full((4, heads_q, dim), largest, dtype=dtype, device=DEV), rand(2, 700, heads_k, dim, dtype=dtype), packed_of(rand(3, 700, heads_k, dim, dtype=dtype))
        q[1] *= 1 - torch.rand(heads_q, dim, generator=g, device=DEV).to(dtype) / 2
        q[2] = -q[2]
        attend_check(q, packed_of(k / 2.0 ** most), v, None)


# ---- far apart ----------------------------------------------------------------------------------------------------------

def test_caches_whose_places_pass_32_bits():
    """Codes, scales and values beyond 2^32 bytes (and 2^31 elements) of where their tensors begin."""
    rows, heads, dim, n = (1 << 23) + 5000, 8, 128, 3000
    for layout in ("head", "row"):
        if layout == "head":
            k, v = (hp.Packed.room(rows, heads, dim, DEV) for _ in range(2))
        else:
            k, v = (hp.Packed(torch.empty(rows, heads, 64, dtype=torch.uint8, device=DEV), torch.empty(rows, heads, 4, 2, dtype=BF16, device=DEV)) for _ in range(2))
        x, y = rand(2, n, heads, dim), rand(3, n, heads, dim)
        hp.hp_pack([x, y], [k.rows(rows - n, rows), v.rows(rows - n, rows)])
        small_k, small_v = packed_of(x), packed_of(y)
        assert torch.equal(k.codes[-n:], small_k.codes) and torch.equal(v.scales[-n:], small_v.scales)
        for q in (rand(1, 3, 16, dim), rand(1, 600, 8, dim)):
            at = torch.arange(len(q), dtype=torch.int32, device=DEV)
            near = torch.stack([at, 2000 + at], 1).contiguous()
            got, want = attend_run(q, k, v, near + (rows - n)), attend_run(q, small_k, small_v, near)
            # the same states in other shares
            exact = plain.attend(q[:3], small_k, small_v, near[:3], dim ** -0.5)
            check("out", got[0][:3], *exact["out"])
            # both are as near to the exact ones: two roundings, and sums of 3000
            apart = (got[0].float() - want[0].float()).abs()
            assert float((apart - 6 * unit(BF16) * (1 + want[0].float().abs())).max()) <= 0
    del k, v
    torch.cuda.empty_cache()
    line = rand(5, 1, heads, dim)
    p = hp.Packed.room(rows, heads, dim, DEV)
    hp.hp_pack([line.expand(rows, heads, dim)], [p])
    one = packed_of(line)
    assert torch.equal(p.codes, one.codes.expand_as(p.codes)) and torch.equal(p.scales, one.scales.expand_as(p.scales))
    back = torch.empty(rows, heads, dim, dtype=BF16, device=DEV)
    hp.hp_unpack([p], [back])
    value = torch.empty_like(line)
    hp.hp_unpack([one], [value])
    assert all(torch.equal(back[a:a + (1 << 20)], value.expand_as(back[a:a + (1 << 20)])) for a in range(0, rows, 1 << 20))


def apart_by(t, stride):
    """The same rows, `stride` elements from one to the next (and of heads what a row has)."""
    far = torch.empty(len(t) * stride, dtype=t.dtype, device=DEV).as_strided(t.shape, (stride, *t[0].contiguous().stride()))
    return far.copy_(t)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_largest_strides(dtype):
    """Rows of a tile of 64 lie 2^30 bytes of codes and 2^31 of scales apart; x beyond what offsets of 32 bits hold takes another way."""
    q, k = rand(1, 3, 4, 96, dtype=dtype), packed_of(rand(2, 130, 2, 96))
    far = hp.Packed(apart_by(k.codes, 1 << 24), apart_by(k.scales, 1 << 24))
    ranges = ranges_of((0, 130), (1, 66), (64, 129))
    got, want = attend_run(q, far, far, ranges), attend_run(q, k, k, ranges)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    w, x = packed_of(rand(3, 130, 320)), rand(4, 40, 320, dtype=dtype)
    far_w = hp.Packed(apart_by(w.codes, 1 << 24), apart_by(w.scales, 1 << 24))
    for rows in (3, 16, 40):
        outs = [torch.empty(rows, 130, dtype=dtype, device=DEV) for _ in range(4)]
        for out, a, b in zip(outs, (x, x, apart_by(x, 1 << 22), apart_by(x, (1 << 22) + 8)), (w, far_w, w, w)):
            hp.hp_packed_linear(a[:rows], b, out)
        assert torch.equal(outs[1], outs[0]) and torch.equal(outs[2], outs[0])
        check("through registers", outs[3], *plain.linear(x[:rows], w))
    with pytest.raises(hp.HpError):
        hp.hp_packed_linear(x, hp.Packed(apart_by(w.codes[:3], (1 << 24) + 16), w.scales[:3]), outs[0][:, :3])


def test_levels_beyond_the_largest_number():
    x = torch.zeros(2, 1, 32, dtype=F32, device=DEV)
    x[0, 0, 3], x[0, 0, 4] = torch.finfo(F32).max, -3.0e38
    x[1, 0, :2] = torch.tensor([3.0e38, 1.0e38])
    p, back = packed_of(x), torch.empty_like(x)
    hp.hp_unpack([p], [back])
    want = plain.values(p, 32)
    fits = want.abs() <= torch.finfo(F32).max
    assert bool(torch.isfinite(p.scales).all()) and torch.equal(back[~fits], torch.full_like(back[~fits], float("inf")))
    check("values", back[fits], want[fits], unit(F32) * want[fits].abs())


# ---- nothing to do --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fast", [None, False])
def test_calls_with_nothing_to_do(monkeypatch, fast):
    monkeypatch.setattr(ops, "_fast", fast)
    for shape in ((0, 3, 64), (5, 0, 64)):
        x = torch.empty(shape, dtype=BF16, device=DEV)
        p = hp.Packed.room(*shape, DEV)
        hp.hp_pack([x], [p])
        hp.hp_unpack([p], [x])
    some, p = rand(1, 5, 2, 64), hp.Packed.room(5, 2, 64, DEV)
    hp.hp_pack([x, some], [hp.Packed.room(5, 0, 64, DEV), p])
    back = torch.empty_like(some)
    hp.hp_unpack([hp.Packed.room(5, 0, 64, DEV), p], [x, back])
    want = plain.values(p, 64)
    check("beside a tensor without heads", back, want, unit(BF16) * want.abs())
    q = torch.empty(0, 4, 64, dtype=BF16, device=DEV)
    assert hp.hp_packed_attend_workspace(q, p) == 0
    hp.hp_packed_attend_step(q, p, p, None, torch.empty_like(q))
    w = hp.Packed.room(7, None, 64, DEV)
    hp.hp_packed_linear(torch.empty(0, 64, dtype=BF16, device=DEV), w, torch.empty(0, 7, dtype=BF16, device=DEV))
    hp.hp_packed_linear(rand(1, 3, 64), hp.Packed.room(0, None, 64, DEV), torch.empty(3, 0, dtype=BF16, device=DEV))
    torch.cuda.synchronize()


# ---- the two ways through the binding -------------------------------------------------------------------------------------

def test_calls_through_python_give_what_the_extension_gives(monkeypatch):
    x, y, m = rand(1, 300, 2, 72), rand(2, 300, 3, 72), rand(3, 40, 100, dtype=F32)
    q, a = rand(4, 7, 6, 72), rand(5, 5, 100, dtype=F32)
    results = []
    for fast in (None, False):
        monkeypatch.setattr(ops, "_fast", fast)
        px, py, pm = hp.Packed.room(300, 2, 72, DEV), hp.Packed.room(300, 3, 72, DEV), hp.Packed.room(40, None, 100, DEV)
        for t in (*px, *py, *pm):
            t.view(torch.uint8).zero_()
        hp.hp_pack([x, y], [px, py])
        hp.hp_pack((m,), (tuple(pm),))
        k, v = packed_of(x), packed_of(rand(6, 300, 2, 72))
        t = dict(bx=torch.empty_like(x), by=torch.empty_like(y), bm=torch.empty_like(m), out=torch.empty_like(q), lse=torch.empty(7, 6, device=DEV),
                 y=torch.empty(5, 40, device=DEV))
        hp.hp_unpack([px, list(py)], [t["bx"], t["by"]])
        hp.hp_unpack([pm], [t["bm"]])
        ws = bytes_of(hp.hp_packed_attend_workspace(q, k))
        hp.hp_packed_attend_step(q, k, list(v), ranges_of(*((i, 300 - i) for i in range(7))), t["out"], lse=t["lse"], scale=0.3, workspace=ws)
        hp.hp_packed_linear(a, pm, t["y"])
        results.append({**t, **{f"{n}{i}": s for n, p in (("px", px), ("py", py), ("pm", pm)) for i, s in enumerate(p)}})
        o, wide = t["out"], hp.Packed(torch.empty(300, 2, 64, dtype=torch.uint8, device=DEV)[:, :, :48], torch.empty(300, 2, 3, 4, dtype=BF16, device=DEV)[..., :2])
        for bad in (lambda: hp.hp_pack([x], [py]), lambda: hp.hp_pack([x, m], [px, pm]), lambda: hp.hp_pack([x, y[:5]], [px, py]), lambda: hp.hp_pack([x.half()], [px]),
                    lambda: hp.hp_pack([x], [px.codes]), lambda: hp.hp_pack([x], [(px.codes, px.scales.float())]), lambda: hp.hp_pack([x], [(px.codes, px.scales[:5])]),
                    lambda: hp.hp_pack([x.transpose(1, 2)], [px]), lambda: hp.hp_unpack([wide], [x]), lambda: hp.hp_unpack([px], [x.float(), x]),
                    lambda: hp.hp_packed_attend_step(q, k, py, None, o, workspace=ws), lambda: hp.hp_packed_attend_step(q[:, :, :64], k, v, None, o, workspace=ws),
                    lambda: hp.hp_packed_attend_step(q, k, v, ranges_of((0, 1)), o, workspace=ws), lambda: hp.hp_packed_attend_step(q, k, v, None, o.float(), workspace=ws),
                    lambda: hp.hp_packed_attend_step(q, x, y, None, o, workspace=ws), lambda: hp.hp_packed_attend_step(q.cpu(), k, v, None, o, workspace=ws),
                    lambda: hp.hp_packed_linear(a[:, :90], pm, t["y"]), lambda: hp.hp_packed_linear(a, px, t["y"]), lambda: hp.hp_packed_linear(a, pm, t["y"][:, :39]),
                    lambda: hp.hp_packed_linear(a, m, t["y"])):
            with pytest.raises((ValueError, TypeError)):
                bad()
        for bad in (lambda: hp.hp_packed_attend_step(q, k, v, None, o), lambda: hp.hp_packed_attend_step(q, k, v, None, o, scale=0.0, workspace=ws),
                    lambda: hp.hp_packed_attend_step(rand(1, 7, 5, 72), k, v, None, rand(1, 7, 5, 72), workspace=ws),
                    lambda: hp.hp_unpack([(torch.zeros(104, dtype=torch.uint8, device=DEV)[8:].view(1, 2, 48), px.scales[:1])], [x[:1]])):
            with pytest.raises(hp.HpError):
                bad()
    for n in results[0]:
        assert torch.equal(results[0][n], results[1][n]), n


# ---- streams and graphs -------------------------------------------------------------------------------------------------

def layer_of(heads_k=2, heads_q=8, dim=64, keys=3000, hidden=512, rows=6):
    """Tensors of a decoding step, and the step: a projection, attention to packed states that new ones join, a projection."""
    t = dict(x=rand(1, rows, hidden), new_k=rand(2, 500, heads_k, dim), new_v=rand(3, 500, heads_k, dim), q=torch.empty(rows, heads_q * dim, dtype=BF16, device=DEV),
             out=torch.empty(rows, heads_q * dim, dtype=BF16, device=DEV), y=torch.empty(rows, hidden, dtype=BF16, device=DEV))
    k, v = packed_of(rand(4, keys, heads_k, dim)), packed_of(rand(5, keys, heads_k, dim))
    wq, wo = packed_of(rand(6, heads_q * dim, hidden, scale=hidden ** -0.5)), packed_of(rand(7, hidden, heads_q * dim, scale=hidden ** -0.5))
    ranges = torch.stack([torch.arange(rows) * 100, torch.full((rows,), keys) - torch.arange(rows) * 50], 1).to(torch.int32).to(DEV).contiguous()

    def step(scratch, stream):
        hp.hp_packed_linear(t["x"], wq, t["q"], stream=stream)
        hp.hp_pack([t["new_k"], t["new_v"]], [k.rows(1000, 1500), v.rows(1000, 1500)], stream=stream)
        hp.hp_packed_attend_step(t["q"].view(rows, heads_q, dim), k, v, ranges, t["out"].view(rows, heads_q, dim), workspace=scratch, stream=stream)
        hp.hp_packed_linear(t["out"], wo, t["y"], stream=stream)
    return t, step, bytes_of(hp.hp_packed_attend_workspace(t["q"].view(rows, heads_q, dim), k)), (k, v, wq, wo, ranges)


def test_a_step_on_another_stream():
    t, step, scratch, _ = layer_of()
    step(scratch, None)
    torch.cuda.synchronize()
    want = t["y"].clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        t["y"].zero_(), t["q"].zero_(), t["out"].zero_()
        side.wait_stream(torch.cuda.current_stream())
        step(scratch, side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(t["y"], want)


def test_two_steps_at_once():
    """On streams of their own, with scratch memory of their own."""
    calls = [layer_of(), layer_of(heads_k=4, dim=128, keys=2500)]
    want = []
    for t, step, scratch, _ in calls:
        step(scratch, None)
        torch.cuda.synchronize()
        want.append(t["y"].clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for t, *_ in calls:
            t["y"].zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for (t, step, scratch, _), stream in zip(calls, streams):
                step(scratch, stream)
        torch.cuda.synchronize()
        assert all(torch.equal(t["y"], y) for (t, *_), y in zip(calls, want))


def test_two_captured_steps_that_share_scratch_memory():
    first, second = layer_of(), layer_of(heads_k=4, dim=128, keys=2500)
    scratch = max(first[2], second[2], key=lambda s: s.numel())
    graphs = []
    side = torch.cuda.Stream()
    for t, step, *_ in (first, second):
        step(scratch, torch.cuda.current_stream())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(scratch, torch.cuda.current_stream())
        graphs.append(graph)
    for i in range(4):
        for t, *_ in (first, second):
            t["x"].copy_(rand(100 + i, *t["x"].shape))
            t["new_v"].copy_(rand(200 + i, *t["new_v"].shape))
            t["y"].zero_()
        for graph in graphs:
            graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        got = [t["y"].clone() for t, *_ in (first, second)]
        for (t, step, *_), y in zip((first, second), got):
            t["y"].zero_()
            step(scratch, torch.cuda.current_stream())
            assert torch.equal(t["y"], y)
            scratch.fill_(0xff)


# ---- together -----------------------------------------------------------------------------------------------------------

def test_a_decoding_step_from_4_bits():
    """Every call on what the one before it made, against the same in 64 bits; the states read back give the plain step."""
    t, step, scratch, (k, v, wq, wo, ranges) = layer_of()
    step(scratch, None)
    check("q", t["q"], *plain.linear(t["x"], wq))
    codes, step_, low = plain.pack(t["new_k"])
    assert torch.equal(k.codes[1000:1500], plain.to_bytes(codes)) and torch.equal(k.scales[1000:1500].double(), torch.stack([step_, low], -1))
    q = t["q"].view(6, 8, 64)
    exact, off = plain.attend(q, k, v, ranges, 64 ** -0.5)["out"]
    check("out", t["out"].view(6, 8, 64), exact, off)
    check("y", t["y"], *plain.linear(t["out"], wo))
    # the same states as values: rounded to bfloat16 once, and 32 bits
    for dtype in (BF16, F32):
        wide_k, wide_v = (torch.empty(3000, 2, 64, dtype=dtype, device=DEV) for _ in range(2))
        out = torch.empty(6, 8, 64, dtype=dtype, device=DEV)
        hp.hp_unpack([k, v], [wide_k, wide_v])
        for p, back in ((k, wide_k), (v, wide_v)):
            want = plain.values(p, 64)
            check("values", back, want, unit(dtype) * want.abs() + 2.0 ** -24 * want.abs())
        qs = q.to(dtype).contiguous()
        hp.hp_cross_attend_step(qs, wide_k, wide_v, ranges, out, workspace=bytes_of(hp.hp_cross_attend_workspace(qs, wide_k, "step")))
        # k's rounding moves scores by at most eps |q| |k|, v's and P's the output by as much of its values
        score = unit(dtype) * 64 ** -0.5 * float((q.double().abs().sum(-1)).max()) * float(wide_k.abs().max())
        most = float(wide_v.abs().max())
        assert float((out.double() - exact).abs().max()) <= 2 * score * most + 4 * unit(dtype) * most + sums(6000) * most


def test_the_example_decodes_from_4_bits():
    """The example's packed step against its plain one with the values that the packed states and weights stand for."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import cross_layer
    hidden, dim, keys, rows = 256, 64, 700, 5
    layer = cross_layer.CrossLayer(hidden, 128, 4, 2, dim, 64, DEV, F32)
    with torch.no_grad():
        k, v = layer.states(rand(1, keys, 128, dtype=F32), torch.arange(2 * keys, dtype=torch.int32, device=DEV).view(2, keys) % 24)
        x, positions = rand(2, rows, hidden, dtype=F32), torch.arange(rows, dtype=torch.int32, device=DEV)
        ranges = ranges_of((0, 700), (3, 4), (5, 5), (100, 165), (1, 650))
        cache, weights = layer.pack(k, v)
        h, z = layer.step_packed(x, positions, *cache, ranges, weights)
        for w, p in zip((layer.wq, layer.wo), weights):
            w.copy_(plain.values(p, w.shape[0]).t())
        want_h, want_z = layer.step(x, positions, *(plain.values(p, dim).to(F32) for p in cache), ranges)
    # two projections, attention and norms in binary32, whose sums cancel by the root of their lengths
    for got, want in ((h, want_h), (z, want_z)):
        assert float((got - want).abs().max()) <= 4 * sums(2 * hidden) * hidden ** 0.5 * float(want.abs().max())
    lines = []
    cross_layer.main(seq=96, side=6, hidden=256, enc_hidden=128, heads_q=4, heads_k=2, steps=1, say=lines.append)
    assert any("4 bits" in line for line in lines)
