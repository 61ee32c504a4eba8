"""The operators of a cross-attention layer in 64 bits, from their definitions, with bounds on what rounding may do.

Every function returns the exact values and, for each, how far a result may be off: half a unit in the last place of
the result's type, and what the roundings on the way there can add up to.  On the way are, for bfloat16, the weights
P and the gradients dS of scores as operands of a product (2^-8 of each: 8 significant bits), and `out` where the backward takes it in;
for binary32 the sums themselves."""
import torch

BF16, F32 = torch.bfloat16, torch.float32


def unit(dtype):
    """Half a unit in the last place, relative: of a result rounded once."""
    return 2.0 ** -8 if dtype is BF16 else 2.0 ** -24


def sums(n):
    """Of a sum of n terms in binary32, relative to the sum of their magnitudes, with room for the functions in them."""
    return (n + 64) * 2.0 ** -24


def rotary(x, table, positions, interleaved, inverse, sections=None):
    """(exact, bound) of one tensor [rows, heads, dim]."""
    half = table.shape[1]
    pos = positions.reshape(-1, x.shape[0]).long()
    axis = torch.cat([torch.full((n,), i) for i, n in enumerate(sections or [half])]).to(x.device)
    inside = (pos >= 0) & (pos < table.shape[0])
    t = table.double()[pos.clamp(0, table.shape[0] - 1)[axis].t(), torch.arange(half, device=x.device)]
    t = torch.where(inside[axis].t()[..., None], t, torch.full_like(t, float("nan")))[:, None]
    c, s = t[..., 0], -t[..., 1] if inverse else t[..., 1]
    y, b = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    xa, xb = x.double()[..., ia], x.double()[..., ib]
    for at, one, two in ((ia, xa * c, -xb * s), (ib, xb * c, xa * s)):
        y[..., at] = one + two
        b[..., at] = unit(x.dtype) * (one + two).abs() + 4 * 2.0 ** -24 * (one.abs() + two.abs())
    return y, b


def norm(x, y, w_post, gate, w_pre, tanh, scale, offset, eps):
    """(h, z) in 64 bits, differentiable; arguments in 64 bits, None where there is none."""
    def normed(t, w):
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * (w + 1 if offset else w)
    h = scale * x
    if y is not None:
        n = y if w_post is None else normed(y, w_post)
        h = h + n * (1 if gate is None else torch.tanh(gate) if tanh else gate)
    return h, (None if w_pre is None else normed(h, w_pre))


def seen(ranges, rows, keys, device):
    j = torch.arange(keys, device=device)
    if ranges is None:
        return torch.ones(rows, keys, dtype=torch.bool, device=device)
    r = ranges.long()
    return (j >= r[:, :1]) & (j < r[:, 1:])


def attend(q, k, v, ranges, scale, dout=None):
    """{name: (exact, bound)} of out, lse and, with dout, dq, dk, dv.  What a row does not see is left out of its sums."""
    dt, (rows, heads_q, dim), (keys, heads_k) = q.dtype, q.shape, k.shape[:2]
    group = heads_q // heads_k
    product, eps = (unit(dt) if dt is BF16 else 0.0), sums(2 * dim)
    mask = seen(ranges, rows, keys, q.device)
    got = {n: [torch.zeros(t, dtype=torch.float64, device=q.device) for _ in range(2)]
           for n, t in (("out", q.shape), ("lse", (rows, heads_q)), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape))}

    def add(name, head, value, bound):
        got[name][0][:, head] += value
        got[name][1][:, head] += bound

    for h in range(heads_q):
        a, b, c = q[:, h].double(), k[:, h // group].double(), v[:, h // group].double()
        s = scale * (a @ b.t().contiguous())
        off = eps * scale * (a.abs() @ b.abs().t().contiguous()) if keys else s        # of a score
        s = s.masked_fill(~mask, float("-inf"))
        lse = torch.logsumexp(s, -1, keepdim=True) if keys else torch.full((rows, 1), float("-inf"), device=q.device).double()
        p = torch.where(mask, torch.exp(s - lse), torch.zeros_like(s))
        # a weight: its rounding, and the exponent's error (the score's, and a few units of the numbers it is made of)
        few = 2.0 ** -21 * (1 + s.masked_fill(~mask, 0).abs() + lse.masked_fill(lse == float("-inf"), 0).abs())
        wide = torch.where(mask, p * (product + 2 * off.masked_fill(~mask, 0) + few + sums(keys)), torch.zeros_like(p))
        cc = torch.where(torch.isfinite(c), c, torch.zeros_like(c)) if keys else c
        o = p @ cc
        ob = wide @ cc.abs() + sums(keys) * (p @ cc.abs())
        add("out", h, o, ob + unit(dt) * o.abs())
        add("lse", h, lse[:, 0], torch.where(torch.isfinite(lse[:, 0]), (wide - product * p).sum(-1) + 2.0 ** -20 * (1 + lse[:, 0].abs()), 0.0))
        if dout is None:
            continue
        g = dout[:, h].double()
        dp = g @ c.t().contiguous()
        delta = (g * o).sum(-1, keepdim=True)
        delta_off = (g.abs() * (ob + unit(dt) * o.abs())).sum(-1, keepdim=True) + sums(dim) * (g * o).abs().sum(-1, keepdim=True)
        ds = torch.where(mask, p * (dp - delta), torch.zeros_like(p))
        # P enters dS unrounded; dS is rounded as an operand
        ds_off = torch.where(mask, (wide - product * p) * (dp - delta).abs() + p * (delta_off + sums(dim) * (g.abs() @ c.abs().t().contiguous())),
                             torch.zeros_like(p)) + product * ds.abs()
        add("dv", h // group, p.t() @ g, wide.t() @ g.abs() + sums(rows * group) * (p.t() @ g.abs()))
        add("dq", h, scale * (ds @ b), scale * (ds_off @ b.abs() + sums(keys) * (ds.abs() @ b.abs())))
        add("dk", h // group, scale * (ds.t() @ a), scale * (ds_off.t() @ a.abs() + sums(rows * group) * (ds.abs().t() @ a.abs())))
    for n in ("dq", "dk", "dv"):
        got[n][1] += unit(dt) * got[n][0].abs()
    return got


def check(name, result, exact, bound, floor=0.0):
    """Asserts |result - exact| <= bound + floor, with NaN and infinities in the same places."""
    r, e = result.double(), exact.double()
    same = torch.isnan(r) == torch.isnan(e)
    assert bool(same.all()), f"{name}: NaN in {int((~same).sum())} wrong places"
    fine = torch.isfinite(e)
    assert torch.equal(r[~fine & ~torch.isnan(e)], e[~fine & ~torch.isnan(e)]), f"{name}: infinities differ"
    # the bounds themselves are to first order: a tenth on top
    over = (r - e).abs() - (1.1 * bound + floor)
    worst = over[fine].max() if bool(fine.any()) else torch.tensor(-1.0)
    assert float(worst) <= 0, f"{name}: {int((over[fine] > 0).sum())} of {r.numel()} values out of bounds, by up to {float(worst):.3g}"
