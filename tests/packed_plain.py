"""States and weights held in 4 bits, in 64 bits from their definitions, with bounds on what rounding may do (see
operators_plain.py).  What rounds on the way: sums in binary32, of codes that are lifted by 16 and of that taken off again;
for bfloat16 the weights P and P * step as operands of a product."""
import torch

from operators_plain import BF16, sums, unit

GROUP = 32


def groups(dim):
    return (dim + GROUP - 1) // GROUP


def bf16_below(x):
    """The largest bfloat16 not above x, in 64 bits (x: 64 bits, finite)."""
    b = x.to(torch.float32)
    b = torch.where(b.double() > x, torch.nextafter(b, torch.full_like(b, float("-inf"))), b)
    i = b.contiguous().view(torch.int32)
    i = torch.where(i < 0, (i + 0xffff) & -65536, i & -65536)
    return i.view(torch.float32).double()


def pack(x):
    """(codes, step, low): [..., groups, 32] whole numbers and [..., groups] in 64 bits, of x [..., dim]."""
    dim = x.shape[-1]
    n = groups(dim)
    codes = torch.zeros(*x.shape[:-1], n, GROUP, dtype=torch.int64, device=x.device)
    step, low = (torch.zeros(*x.shape[:-1], n, dtype=torch.float64, device=x.device) for _ in range(2))
    for g in range(n):
        v = x[..., g * GROUP:(g + 1) * GROUP].double()
        fine = (v.abs() <= torch.finfo(torch.float32).max).all(-1) & (v >= -torch.finfo(BF16).max).all(-1)
        v = torch.where(fine[..., None], v, torch.zeros_like(v))
        lo = bf16_below(v.amin(-1))
        d = (v.amax(-1) - lo) / 15
        s = torch.where(d < 2.0 ** -126, torch.zeros_like(d), -bf16_below(-d))
        level = torch.arange(15, device=x.device).double() + 0.5
        c = ((v - lo[..., None])[..., None] > level * s[..., None, None]).sum(-1)
        c = torch.where(((s == 0) | ~fine)[..., None], torch.zeros_like(c), c)
        codes[..., g, :v.shape[-1]] = c
        nan = torch.full_like(s, float("nan"))
        step[..., g], low[..., g] = torch.where(fine, s, nan), torch.where(fine, lo, nan)
    return codes, step, low


def to_bytes(codes):
    """Codes [..., groups, 32] as they lie in memory, uint8 [..., 16 * groups]."""
    c = codes.flatten(-2)
    out = torch.zeros(*c.shape[:-1], c.shape[-1] // 2, dtype=torch.int64, device=c.device)
    for word in range(c.shape[-1] // 8):
        for i in range(4):
            for half in range(2):
                bit = 4 * i + 16 * half
                out[..., 4 * word + bit // 8] += c[..., 8 * word + 2 * i + half] << (bit % 8)
    return out.to(torch.uint8)


def from_bytes(data):
    """[..., groups, 32] of uint8 [..., 16 * groups]."""
    b = data.long()
    out = torch.zeros(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.int64, device=b.device)
    for word in range(b.shape[-1] // 4):
        for i in range(4):
            for half in range(2):
                bit = 4 * i + 16 * half
                out[..., 8 * word + 2 * i + half] = b[..., 4 * word + bit // 8] >> (bit % 8) & 15
    return out.unflatten(-1, (-1, GROUP))


def parts(packed, dim):
    """(code, step, low) of each channel, [..., dim] in 64 bits, of a pair (codes, scales)."""
    c = from_bytes(packed[0]).double().flatten(-2)[..., :dim]
    s = packed[1].double().repeat_interleave(GROUP, -2)[..., :dim, :]
    return c, s[..., 0], s[..., 1]


def values(packed, dim):
    c, step, low = parts(packed, dim)
    return low + step * c


def linear(x, packed):
    """(exact, bound) of x times the transpose of a packed matrix."""
    c, step, low = parts(packed, x.shape[1])
    w, most = low + step * c, low.abs() + 47 * step
    o = x.double() @ w.t().contiguous()
    return o, unit(x.dtype) * o.abs() + sums(2 * x.shape[1]) * (x.double().abs() @ most.t().contiguous())


def attend(q, k, v, ranges, scale):
    """{name: (exact, bound)} of out and lse, row by row.  What a row does not see is not looked at."""
    dt, (rows, heads_q, dim), (keys, heads_k) = q.dtype, q.shape, k[0].shape[:2]
    group, rounding = heads_q // heads_k, (unit(dt) if dt is BF16 else 2.0 ** -24)
    out, off_out = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    lse, off_lse = (torch.zeros(rows, heads_q, dtype=torch.float64, device=q.device) for _ in range(2))
    for r in range(rows):
        a, b = (0, keys) if ranges is None else (max(0, int(ranges[r, 0])), min(keys, int(ranges[r, 1])))
        if a >= b:
            lse[r] = float("-inf")
            continue
        n = b - a
        kc, ks, kl = parts((k[0][a:b], k[1][a:b]), dim)
        vc, vs, vl = parts((v[0][a:b], v[1][a:b]), dim)
        for h in range(heads_q):
            j, x = h // group, q[r, h].double()
            s = scale * ((kl + ks * kc)[:, j] @ x)
            off = scale * sums(2 * dim) * ((kl.abs() + 47 * ks)[:, j] @ x.abs())
            total = torch.logsumexp(s, 0)
            p = torch.exp(s - total)
            few = 2.0 ** -21 * (1 + s.abs() + total.abs())
            wide = p * (2 * off + few + sums(n))
            o = p @ (vl + vs * vc)[:, j]
            out[r, h] = o
            off_out[r, h] = (wide @ (vl + vs * vc)[:, j].abs() + rounding * (p @ ((vs * (vc - 8)).abs() + (vl + 8 * vs).abs())[:, j])
                             + sums(2 * n) * (p @ (vl.abs() + 63 * vs)[:, j]) + unit(dt) * o.abs())
            lse[r, h] = total
            off_lse[r, h] = wide.sum() + 2.0 ** -20 * (1 + total.abs())
    return {"out": (out, off_out), "lse": (lse, off_lse)}
