"""Places of the operators where waves meet, values cancel or arguments only nearly fit, on the GPU."""
import pytest
import torch

import operators_plain as plain
import paper_2605_27678_amd as hp
from operators_plain import BF16, F32, check
from paper_2605_27678_amd import operators as ops

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def rand(seed, *shape, dtype=BF16):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def whole(seed, low, high, *shape):
    """Whole numbers from low to high."""
    return torch.randint(low, high + 1, shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(BF16)


def bytes_of(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=DEV)


def attend_run(q, k, v, ranges, dout=None, scale=None, step=False):
    rows, heads_q, _ = q.shape
    got = {"out": torch.full_like(q, 7.0), "lse": torch.full((rows, heads_q), 7.0, dtype=F32, device=DEV)}
    call = hp.hp_cross_attend_step if step else hp.hp_cross_attend
    call(q, k, v, ranges, got["out"], lse=got["lse"], scale=scale, workspace=bytes_of(hp.hp_cross_attend_workspace(q, k, "step" if step else "forward")))
    if dout is not None:
        got.update({n: torch.full_like(t, 7.0) for n, t in (("dq", q), ("dk", k), ("dv", v))})
        hp.hp_cross_attend_backward(q, k, v, ranges, got["out"], got["lse"], dout, got["dq"], got["dk"], got["dv"], scale=scale,
                                    workspace=bytes_of(hp.hp_cross_attend_workspace(q, k, "backward")))
    return got


# ---- where waves meet ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dim", [64, 72, 80, 88, 96, 128, 256])
def test_gradients_of_states_over_a_hundred_tiles_a_part(dim):
    """Every tile of rows counts, and exactly: keys of zeros give each of 2048 states the weight 2^-11, values that come in
    pairs of a number and its negative give out = 0, and all else is whole numbers, so that dv = 2^-11 sum dout and
    dk = scale 2^-11 sum (dout . v) q are whole multiples of a power of two, whatever the order of their sums, and are
    rounded once.  A piece of another tile in a sum would change it."""
    rows, keys, heads_q, heads_k, scale = 16384, 2048, 32, 16, 0.125
    q, dout = whole(1, -3, 3, rows, heads_q, dim), whole(2, -3, 3, rows, heads_q, dim)
    k = torch.zeros(keys, heads_k, dim, dtype=BF16, device=DEV)
    v = torch.zeros_like(k)
    v[: keys // 2, :, 1:dim:13] = whole(3, -2, 2, keys // 2, heads_k, len(range(1, dim, 13)))
    v[keys // 2:] = -v[: keys // 2]
    got = attend_run(q, k, v, None, dout, scale)
    assert not bool(got["out"].any()) and not bool(got["dq"].any())
    group = heads_q // heads_k
    for h in range(heads_k):
        a, g = (t[:, h * group:(h + 1) * group].reshape(-1, dim).double() for t in (q, dout))
        dp = g @ v[:, h].double().t().contiguous()
        assert float(dp.abs().max()) <= 256                              # as bfloat16 holds them
        dv, dk = g.sum(0) / keys, scale / keys * (dp.t().contiguous() @ a)
        assert torch.equal(got["dv"][:, h], dv.to(BF16).expand(keys, dim)), f"dv of head {h}"
        assert torch.equal(got["dk"][:, h], dk.to(BF16)), f"dk of head {h}"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_workgroups_that_begin_again_do_so_whole(dim, dtype):
    """Samples of 48 rows and 80 states, so that every workgroup has tiles that not all of its rows see; one sample in two
    holds values that are not finite, and the others' results are those of the calls without them."""
    n, heads_q, heads_k = 40, 4, 2
    rows, keys = 48 * n, 80 * n
    q, k, v, dout = (rand(i, m, h, dim, dtype=dtype) for i, (m, h) in enumerate(((rows, heads_q), (keys, heads_k), (keys, heads_k), (rows, heads_q))))
    sample = torch.arange(rows, device=DEV) // 48
    ranges = torch.stack([80 * sample, 80 * (sample + 1)], 1).to(torch.int32)
    good = attend_run(q, k, v, ranges, dout)
    for t, each in ((q, 48), (dout, 48), (k, 80), (v, 80)):
        part = t.view(n, each, *t.shape[1:])
        part[1::2, ::7], part[1::2, 3::7] = float("nan"), float("inf")
    for turn in range(3):
        got = attend_run(q, k, v, ranges, dout)
        for name, t in got.items():
            a, b = (x.view(n, -1, *x.shape[1:])[::2].double() for x in (t, good[name]))
            assert bool(torch.isfinite(a).all()), (turn, name)
            # value by value instead of by matrix products: other sums of the same terms
            off = 2 * plain.unit(dtype) * b.abs() + 2.0 ** -8 * (1 if dtype is BF16 else 2.0 ** -12)
            assert bool(((a - b).abs() <= off).all()), (turn, name)


# ---- where values cancel ------------------------------------------------------------------------------------------------

def gate_gradient(x, y, w_post, gate, w_pre, scale, dh, dz, eps=1e-6):
    """(exact, bound) of the gradient of tanh(gate) in 64 bits: sums over rows (and channels, for one gate) of
    D y r1 w1 slope, slope = 1 - tanh^2 = (2 / (e^g + e^-g))^2.  A term is a few products of numbers that carry the roundings
    of sums over a row - a lane's up to 64 values, six steps over a wave, 16 waves - and passes, on its way, its group's
    rows, every 32nd line, 32 of these sums and, for one gate, every 1024th channel and 21 more."""
    a, b, w1, w2, g = (t.double() for t in (x, y, w_post, w_pre, gate))
    slope = (2 / (g.exp() + (-g).exp())).square()
    r1 = 1 / (b.square().mean(-1, keepdim=True) + eps).sqrt()
    n = b * r1 * w1
    h = scale * a + g.tanh() * n
    r2 = 1 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    d = dz.double() * w2 * r2
    whole = dh.double() + d - h * r2.square() * (h * d).mean(-1, keepdim=True)
    most = dh.double().abs() + d.abs() + h.abs() * r2.square() * (h * d).abs().mean(-1, keepdim=True)
    e, m = (whole * n).sum(0) * slope, (most * n.abs()).sum(0) * slope
    if gate.numel() == 1:
        e, m = e.sum().view(1), m.sum().view(1)
    rows, hidden = x.shape
    ways = 8 * plain.sums(86) + plain.sums(rows // 256 + rows // 32 + 33 + hidden // 1024 + 24)
    return e, plain.unit(x.dtype) * e.abs() + ways * m


def gate_case(rows, hidden, dtype, gate):
    """The whole gradient of a training step, with dh along the block's output so that the sum for one gate does not cancel."""
    x, y, dz = rand(1, rows, hidden, dtype=dtype), rand(2, rows, hidden, dtype=dtype), rand(4, rows, hidden, dtype=dtype)
    dh = (y.float() + 0.5 * rand(3, rows, hidden, dtype=F32)).to(dtype)
    w1, w2 = (1 + 0.1 * rand(5 + i, hidden, dtype=F32).to(dtype) for i in range(2))
    h, z, dx, dy = (torch.empty_like(x) for _ in range(4))
    rstd, dgate = torch.empty(2, rows, dtype=F32, device=DEV), torch.full_like(gate, 7.0)
    hp.hp_gated_norm(x, y, h, z, w1, gate, w2, gate_tanh=True, residual_scale=0.5, rstd=rstd)
    hp.hp_gated_norm_backward(dh, dz, x, y, rstd, w1, gate, w2, dx, dy, None, dgate, None, gate_tanh=True, residual_scale=0.5,
                              workspace=bytes_of(hp.hp_gated_norm_workspace(rows, hidden)))
    return (dgate, *gate_gradient(x, y, w1, gate, w2, 0.5, dh, dz))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", [0.0, 0.25, -1.0, 4.0, -8.0, 12.0, -40.0, 100.0])
def test_the_gradient_of_a_gate_far_from_zero(gate, dtype):
    for size in (1, 328):
        dgate, exact, bound = gate_case(37, 328, dtype, torch.full((size,), gate, dtype=dtype, device=DEV))
        check(f"dgate of {size}", dgate, exact, bound, 1e-37)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,hidden", [(1, 64), (3, 7), (65, 512), (33, 1000), (5, 2305), (300, 4096), (17, 5120), (2500, 512), (6, 8193),
                                         (700, 12288), (2, 32768)])
def test_the_gradient_of_one_gate_for_all_channels(rows, hidden, dtype):
    dgate, exact, bound = gate_case(rows, hidden, dtype, torch.full((1,), 0.75, dtype=dtype, device=DEV))
    # what a gradient without the slope (0.60 here), or of nine rows in ten, would be is out of bounds
    assert float(bound) < 0.05 * float(exact.abs())
    check("dgate", dgate, exact, bound)


# ---- arguments that only nearly fit ---------------------------------------------------------------------------------------

@pytest.fixture(params=["extension", "python"])
def way(request, monkeypatch):
    """Calls by the extension, and by Python, which takes what the extension leaves to it."""
    if request.param == "python":
        monkeypatch.setattr(ops, "_fast", False)


def test_a_gate_without_values_is_no_missing_gate(way):
    x, y, w, none = rand(1, 5, 64), rand(2, 5, 64), torch.ones(64, dtype=BF16, device=DEV), torch.empty(0, dtype=BF16, device=DEV)
    h, z, rstd = torch.full_like(x, 7.0), torch.full_like(x, 7.0), torch.full((2, 5), 7.0, device=DEV)
    with pytest.raises(ValueError, match="gate"):
        hp.hp_gated_norm(x, y, h, z, w, none, w, rstd=rstd)
    dx, dy = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    with pytest.raises(ValueError, match="gate"):
        hp.hp_gated_norm_backward(x, y, x, y, rstd, w, none, w, dx, dy, None, None, None)
    with pytest.raises(ValueError, match="gate"):
        hp.gated_norm(x, y, w, none, w)
    for t in (h, z, dx, dy, rstd):
        assert bool((t == 7.0).all())


def test_switches_that_are_neither_true_nor_false(way):
    x, table = rand(1, 5, 2, 16), torch.ones(8, 8, 2, device=DEV)
    pos, out, both = torch.arange(5, dtype=torch.int32, device=DEV), torch.full((5, 2, 16), 7.0, dtype=BF16, device=DEV), torch.tensor([True, False])
    for how in (dict(interleaved=both), dict(inverse=both), dict(interleaved=both, inverse=both)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            hp.hp_rotary([x], [out], table, pos, **how)
    w, h = torch.ones(16, dtype=BF16, device=DEV), torch.full((5, 16), 7.0, dtype=BF16, device=DEV)
    for how in (dict(gate_tanh=both), dict(unit_offset=both)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            hp.hp_gated_norm(x[:, 0], x[:, 1], h, None, w, **how)
    assert bool((out == 7.0).all()) and bool((h == 7.0).all())
