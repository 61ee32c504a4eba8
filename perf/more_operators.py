"""The operators of a cross-attention layer that serves from 4 bits, as cases that can be timed and checked.

Decoding reads, for every token, the encoder's states that a request keeps and the projections' weights.  Both are
held packed here: groups of 32 neighbouring channels with a code of 4 bits a value and a step and a low value for the
group, value = low + step * code.

  cache    states of images packed as they are written (k and v in one call), and read back as values
  attend   one token of each of several requests against its own stretch of a packed cache
  linear   a few rows times a packed weight matrix, out = x W^T

The packed form: [rows, heads, channels] become codes, uint8 [rows, heads, 16 * groups], and scales, bfloat16 [rows,
heads, groups, 2] (step, low); matrices have no heads.  A group's 16 bytes are four little-endian 32-bit words; word w
has channel 8w + 2i in bits 4i to 4i + 3 and channel 8w + 2i + 1 in bits 16 + 4i to 19 + 4i.  low is the largest
bfloat16 not above the least value, step the least bfloat16 not below (greatest - low) / 15, and a value's code is
that of the nearest level, of the lower one of two.

Sizes are those of the library's workloads (hidden 64 to 12288, images of 16 to 4096 tokens, sequences up to 131072,
TP 1 to 8) in heads of 64 to 256 channels.  Keys have channels that stand apart, as keys do; activations are normalised
with a few large channels; weights are N(0, 1 / inputs) with rows of different sizes.

`own` false: plain torch operations in 32 bits (64 where codes are decided), rounded once at the end.  `own` true: the
library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
GROUP = 32

FIELDS = dict(op="", f32=False,
              # cache and attend
              heads_q=0, heads_k=0, dim=128,
              # cache: states; linear: rows of activations
              rows=0,
              # attend: requests with len_lo to len_hi states, in a cache with `spare` rows between them
              requests=0, len_lo=0, len_hi=0, spare=0,
              # linear
              n_in=0, n_out=0)

MOST_BYTES = 4.2e8
MOST_CACHE = 83e6            # values of k and v
MOST_WEIGHTS = 152e6
MOST_PRODUCTS = 1.0e10       # rows x weights
MOST_STATES = 260e6          # values of k (v has as many)


def _case(name=None, **kw):
    c = dict(FIELDS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one image's states join a request's cache
        _case("cache_image", op="cache", rows=576, heads_k=8),
        # the long-context workload's 40139 states on one rank of TP 1
        _case("cache_long", op="cache", rows=40139, heads_k=8),
        # an encoder's own heads of 72 channels, binary32, an odd number of states
        _case("cache_odd_f32", op="cache", f32=True, rows=5761, heads_k=16, dim=72),
        # decoding: one request with one image
        _case("attend_one", op="attend", heads_q=32, heads_k=8, requests=1, len_lo=576, len_hi=576),
        # decoding: 64 requests with 1 to 11 images each, TP 1 of 64 heads
        _case("attend_batch", op="attend", heads_q=64, heads_k=8, requests=64, len_lo=576, len_hi=6404, spare=37),
        # two long videos, heads of 256 channels
        _case("attend_long", op="attend", heads_q=16, heads_k=2, dim=256, requests=2, len_lo=40139, len_hi=131072),
        # ragged requests, heads of 72 channels with a state head each, binary32
        _case("attend_odd_f32", op="attend", f32=True, heads_q=16, heads_k=16, dim=72, requests=30, len_lo=1,
              len_hi=2305, spare=1),
        # decoding: one token's projection
        _case("linear_one", op="linear", rows=1, n_in=4096, n_out=4096),
        # decoding: 16 tokens at hidden 12288
        _case("linear_wide", op="linear", rows=16, n_in=12288, n_out=12288),
        # decoding: 64 tokens at hidden 8192
        _case("linear_batch", op="linear", rows=64, n_in=8192, n_out=8192),
        # sizes that no tile divides, binary32
        _case("linear_odd_f32", op="linear", f32=True, rows=5, n_in=2305, n_out=5121),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        if c is not None and work(c)["bytes"] <= MOST_BYTES:
            return c


def _draw(rng):
    op = rng.choice(["cache", "attend", "attend", "linear", "linear"])
    f32 = rng.random() < 0.25
    if op == "linear":
        n_in, n_out = _log(rng, 64, 16384), _log(rng, 16, 49152)
        if rng.random() < 0.6:                               # most projections are of whole tiles
            n_in, n_out = max(1, round(n_in / 128)) * 128, max(1, round(n_out / 64)) * 64
        rows = _log(rng, 1, 128)
        if n_in * n_out > MOST_WEIGHTS or rows * n_in * n_out > MOST_PRODUCTS:
            return None
        return _case(op=op, f32=f32, rows=rows, n_in=n_in, n_out=n_out)
    dim = rng.choice([64, 72, 80, 96, 128, 128, 128, 256])
    heads_k = rng.choice([1, 2, 4, 8, 16])
    if op == "cache":
        rows = _log(rng, 1, 131072)
        if 2 * rows * heads_k * dim > MOST_CACHE / (2 if f32 else 1):
            return None
        return _case(op=op, f32=f32, rows=rows, heads_k=heads_k, dim=dim)
    heads_q = heads_k * rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
    lo = _log(rng, 1, 4000)
    hi = _log(rng, lo, 131072)
    requests = _log(rng, 1, 256)
    if requests * (lo + hi) / 2 * heads_k * dim > MOST_STATES or heads_q > 128:
        return None
    return _case(op=op, f32=f32, dim=dim, heads_q=heads_q, heads_k=heads_k, requests=requests, len_lo=lo, len_hi=hi,
                 spare=rng.choice([0, 1, 37]))


# ---- the packed form ---------------------------------------------------------------------------------------

def _groups(dim):
    return (dim + GROUP - 1) // GROUP


def _grouped(x):
    """[..., dim] -> [..., groups, 32]; the last channel stands for those that a shorter last group lacks."""
    dim = x.shape[-1]
    lack = _groups(dim) * GROUP - dim
    if lack:
        x = torch.cat([x, x[..., -1:].expand(*x.shape[:-1], lack)], -1)
    return x.unflatten(-1, (-1, GROUP))


def _bits_down(x):
    """The largest bfloat16 not above x (binary32), as binary32."""
    b = x.contiguous().view(torch.int32)
    return torch.where(b < 0, (b + 0xffff) & -65536, b & -65536).view(torch.float32)


def _bits_up(x):
    """The least bfloat16 not below x (64 bits, not negative), as binary32."""
    f = x.float()
    f = torch.where(f.double() < x, torch.nextafter(f, torch.full_like(f, float("inf"))), f)
    return ((f.view(torch.int32) + 0xffff) & -65536).view(torch.float32)


def _plain_codes(x):
    """(codes 0 to 15 [..., groups, 32], step, low [..., groups, 1] in binary32) of x [..., dim]."""
    g = _grouped(x.float())
    low = _bits_down(g.amin(-1, keepdim=True))
    d = (g.amax(-1, keepdim=True).double() - low.double()) / 15.0
    step = _bits_up(torch.where(d < 2.0 ** -126, torch.zeros_like(d), d))
    t = (g.double() - low.double()) / torch.where(step == 0, torch.ones_like(step), step).double()
    return torch.ceil(t - 0.5).clamp_(0, 15).to(torch.uint8), step, low


def _words(codes, dim):
    """Codes [..., groups, 32] as bytes [..., 16 * groups]."""
    codes = codes.flatten(-2)
    codes[..., dim:] = 0
    c = codes.unflatten(-1, (-1, 4, 2)).int()                  # [..., words, i, channel of a pair]
    shift = torch.arange(4, device=c.device, dtype=torch.int32) * 4
    half = (c << shift[:, None]).sum(-2).to(torch.int32)       # [..., words, 2]: the halves of a word
    return torch.stack([half & 255, half >> 8], -1).flatten(-3).to(torch.uint8)


def _pack(x, codes, scales):
    """x [rows, (heads,) dim] into codes and scales, some rows at a time."""
    each = max(1, (1 << 24) // max(1, x[0].numel()))
    for a in range(0, x.shape[0], each):
        c, step, low = _plain_codes(x[a:a + each])
        codes[a:a + each] = _words(c, x.shape[-1])
        scales[a:a + each] = torch.cat([step, low], -1).to(torch.bfloat16)


def _values(codes, scales, dim):
    """The values that packed rows stand for, binary32 [..., dim]."""
    b = codes.int().unflatten(-1, (-1, 2, 2))                  # [..., words, half, byte]
    half = b[..., 0] | b[..., 1] << 8                          # [..., words, half]
    shift = torch.arange(4, device=b.device, dtype=torch.int32) * 4
    c = (half[..., None, :] >> shift[:, None]) & 15            # [..., words, i, half]
    s = scales.float()
    return (c.flatten(-3).unflatten(-1, (-1, GROUP)).float() * s[..., :1] + s[..., 1:]).flatten(-2)[..., :dim]


def _room(rows, heads, dim):
    """Room for packed rows: the stretch of a head is in one piece, and so is its scales'."""
    g = _groups(dim)
    return (torch.empty(heads, rows, 16 * g, dtype=torch.uint8, device=DEV).transpose(0, 1),
            torch.empty(heads, rows, g, 2, dtype=torch.bfloat16, device=DEV).transpose(0, 1))


# ---- inputs ----------------------------------------------------------------------------------------------

def _stretches(c):
    """First and end of each request's states, and how many rows the cache has."""
    n = c["requests"]
    lens = [c["len_lo"] + (c["len_hi"] - c["len_lo"]) * (i * 7919 % n) // max(1, n - 1) for i in range(n)]
    starts = np.cumsum([0] + [x + c["spare"] for x in lens])
    return np.stack([starts[:n], starts[:n] + np.array(lens)], 1).astype(np.int32), int(starts[n])


def _states(c, rows, g, dt):
    """k and v of `rows` states: keys have a place of their own for each channel, and some channels are large."""
    shape = (c["heads_k"], c["dim"])
    at, size = torch.randn(shape, generator=g, device=DEV), 0.5 + torch.rand(shape, generator=g, device=DEV)
    size = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.03, 3 * size, size)
    k = (torch.randn((rows, *shape), generator=g, device=DEV).mul_(size).add_(at)).to(dt)
    v = torch.randn((rows, *shape), generator=g, dtype=dt, device=DEV)
    return k, v


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed) + 31)
    dt = torch.float32 if c["f32"] else torch.bfloat16
    s = {"case": c}
    if c["op"] == "linear":
        w = torch.randn((c["n_out"], c["n_in"]), generator=g, device=DEV) / c["n_in"] ** 0.5
        w *= 0.5 + torch.rand((c["n_out"], 1), generator=g, device=DEV)
        n = _groups(c["n_in"])
        s["w"] = (torch.empty(c["n_out"], 16 * n, dtype=torch.uint8, device=DEV),
                  torch.empty(c["n_out"], n, 2, dtype=torch.bfloat16, device=DEV))
        _pack(w.to(dt), *s["w"])
        x = torch.randn((c["rows"], c["n_in"]), generator=g, device=DEV)
        large = torch.rand(c["n_in"], generator=g, device=DEV) < 0.01
        s["x"] = torch.where(large, 8 * x, x).to(dt)
        s["out"] = torch.empty(c["rows"], c["n_out"], dtype=dt, device=DEV)
    elif c["op"] == "cache":
        s["x"] = list(_states(c, c["rows"], g, dt))
        s["packed"] = [_room(c["rows"], c["heads_k"], c["dim"]) for _ in s["x"]]
        s["out"] = [torch.empty_like(x) for x in s["x"]]
    else:
        ranges, rows = _stretches(c)
        s["ranges"] = torch.from_numpy(ranges).to(DEV)
        s["q"] = torch.randn((c["requests"], c["heads_q"], c["dim"]), generator=g, dtype=dt, device=DEV)
        s["k"], s["v"] = _room(rows, c["heads_k"], c["dim"]), _room(rows, c["heads_k"], c["dim"])
        for to, x in zip((s["k"], s["v"]), _states(c, rows, g, dt)):
            _pack(x, *to)
        s["out"] = torch.empty_like(s["q"])
    return s


# ---- one pass --------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2605_27678_amd as hp
        return {"cache": _own_cache, "attend": _own_attend, "linear": _own_linear}[op](hp, s)
    return {"cache": _plain_cache, "attend": _plain_attend, "linear": _plain_linear}[op](s)


def _own_cache(hp, s):
    hp.hp_pack(s["x"], s["packed"])
    hp.hp_unpack(s["packed"], s["out"])
    return s["out"]


def _own_attend(hp, s):
    if "workspace" not in s:                                 # as a program allocates once for its shapes
        s["workspace"] = torch.empty(hp.hp_packed_attend_workspace(s["q"], s["k"]), dtype=torch.uint8, device=DEV)
    hp.hp_packed_attend_step(s["q"], s["k"], s["v"], s["ranges"], s["out"], workspace=s["workspace"])
    return s["out"]


def _own_linear(hp, s):
    hp.hp_packed_linear(s["x"], s["w"], s["out"])
    return s["out"]


def _plain_cache(s):
    dim = s["case"]["dim"]
    for x, (codes, scales) in zip(s["x"], s["packed"]):
        _pack(x, codes, scales)
    return [_values(codes, scales, dim).to(x.dtype) for x, (codes, scales) in zip(s["x"], s["packed"])]


def _plain_attend(s):
    c, q = s["case"], s["q"]
    heads_k, dim = c["heads_k"], c["dim"]
    out = torch.empty_like(q)
    ranges, _ = _stretches(c)
    for i, (a, b) in enumerate(ranges.tolist()):
        k = _values(s["k"][0][a:b], s["k"][1][a:b], dim).permute(1, 2, 0).contiguous()
        v = _values(s["v"][0][a:b], s["v"][1][a:b], dim).permute(1, 0, 2).contiguous()
        p = torch.matmul(q[i].float().view(heads_k, -1, dim), k) * (1.0 / math.sqrt(dim))
        p = (p - p.amax(-1, keepdim=True)).exp()
        out[i] = (torch.matmul(p, v) / p.sum(-1, keepdim=True)).reshape(-1, dim).to(q.dtype)
    return out


def _plain_linear(s):
    w = _values(*s["w"], s["case"]["n_in"])
    return torch.matmul(s["x"].float(), w.t()).to(s["x"].dtype)


# ---- what a pass cannot do without -------------------------------------------------------------------------

def work(case):
    c, e = case, 4 if case["f32"] else 2
    if c["op"] == "linear":
        weights = c["n_out"] * (c["n_in"] / 2 + 4 * _groups(c["n_in"]))
        return {"bytes": int(weights) + c["rows"] * (c["n_in"] + c["n_out"]) * e,
                "flops": 2 * c["rows"] * c["n_in"] * c["n_out"]}
    packed = 2 * c["heads_k"] * (c["dim"] / 2 + 4 * _groups(c["dim"]))       # bytes of a state's k and v
    if c["op"] == "cache":
        values = 2 * c["rows"] * c["heads_k"] * c["dim"]
        return {"bytes": int(2 * values * e + 2 * c["rows"] * packed), "flops": 6 * values}
    r, _ = _stretches(c)
    seen = int((r[:, 1].astype(np.int64) - r[:, 0]).sum())
    return {"bytes": int(seen * packed) + 2 * c["requests"] * c["heads_q"] * c["dim"] * e,
            "flops": 4 * seen * c["heads_q"] * c["dim"]}


# ---- in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"cache": _exact_cache, "attend": _exact_attend, "linear": _exact_linear}[case["op"]](s)


def _levels(codes, scales, dim):
    """[..., dim] in 64 bits: each value looked up among its group's sixteen levels."""
    out = torch.empty(*codes.shape[:-1], _groups(dim) * GROUP, dtype=torch.float64, device=DEV)
    s = scales.double()
    levels = s[..., 1:] + s[..., :1] * torch.arange(16, device=DEV).double()
    for c in range(GROUP):                                   # the byte and the half of it that channel c is in
        w, i, high = c // 8, c % 8 // 2, c % 2
        byte = codes[..., 4 * w + 2 * high + i // 2::16].long()
        code = byte % 16 if i % 2 == 0 else byte // 16
        out[..., c::GROUP] = levels.gather(-1, code[..., None])[..., 0]
    return out[..., :dim]


def _exact_cache(s):
    """Group by group: the levels from the greatest and least value, and the level that is nearest."""
    out = []
    for x in s["x"]:
        y, dim = torch.empty(x.shape, dtype=torch.float64, device=DEV), x.shape[-1]
        for a in range(0, dim, GROUP):
            g = x[..., a:a + GROUP].double()
            least, greatest = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
            low = least.to(torch.bfloat16)
            low = torch.where(low.double() > least, _next(low, -1), low).double()
            step = ((greatest - low) / 15).to(torch.bfloat16)
            step = torch.where(step.double() < (greatest - low) / 15, _next(step, 1), step).double()
            step = torch.where((greatest - low) / 15 < 2.0 ** -126, torch.zeros_like(step), step)
            n = torch.zeros_like(g)
            for k in range(15):
                n += g - low > (k + 0.5) * step
            y[..., a:a + GROUP] = low + step * torch.where(step == 0, torch.zeros_like(n), n)
        out.append(y)
    return out


def _next(x, way):
    """The bfloat16 above (way 1) or below (way -1)."""
    f = x.float().double()
    size = torch.maximum(torch.exp2(torch.floor(torch.log2(f.abs().clamp(min=2.0 ** -126))) - 7), torch.full_like(f, 2.0 ** -133))
    toward = f + way * size
    # at a power of two the numbers towards zero lie twice as close
    closer = f + way * size / 2
    return torch.where(closer.to(torch.bfloat16).double() == closer, closer, toward).to(torch.bfloat16)


def _exact_attend(s):
    c, q = s["case"], s["q"].double()
    dim, group = c["dim"], c["heads_q"] // c["heads_k"]
    out = torch.zeros_like(q)
    for i, (a, b) in enumerate(s["ranges"].tolist()):
        for h in range(c["heads_k"]):
            k = _levels(s["k"][0][a:b, h], s["k"][1][a:b, h], dim)
            v = _levels(s["v"][0][a:b, h], s["v"][1][a:b, h], dim)
            of = slice(h * group, (h + 1) * group)
            w = torch.softmax(torch.matmul(k, q[i, of].t().contiguous()) / dim ** 0.5, 0)
            out[i, of] = torch.matmul(w.t().contiguous(), v)
    return out


def _exact_linear(s):
    c = s["case"]
    out = torch.empty(c["rows"], c["n_out"], dtype=torch.float64, device=DEV)
    x = s["x"].double()
    for a in range(0, c["n_out"], 2048):
        w = _levels(s["w"][0][a:a + 2048], s["w"][1][a:a + 2048], c["n_in"])
        out[:, a:a + 2048] = torch.matmul(x, w.t().contiguous())
    return out
