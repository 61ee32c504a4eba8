"""The operators of a cross-attention layer over a boundary, as cases that can be timed and checked.

A language model takes an encoder's tokens either into its own sequence (the boundary transform) or through layers
whose queries attend to the encoder's states.  Such a layer is made of the operators measured here, between its
projections:

  rotary        positions turned into the heads of queries and keys: halves or interleaved pairs, part of a head,
                one position a row or one for each axis of a grid; `inverse` is the gradient
  norm          h = residual_scale * x + gate * norm(y), z = norm(h): the block output y joins the residual stream
                and the next block's input comes out, forward alone or with every gradient
  attend        attention of packed query rows to packed encoder states; each row sees a range of them, here the
                images of its sample that ended before it, so that rows before the first image see nothing
  attend_train  the same with the gradients of q, k and v
  attend_step   one token of each of several requests against its own stretch of a cache of encoder states

Sizes are those of the library's workloads (hidden 64 to 12288, images of 16 to 4096 tokens, sequences up to
131072, TP 1 to 8, CP 1 to 8) in heads of 64 to 256 channels.  Values are N(0, 1), as normalised activations and
scaled gradients are; weights of norms lie around one, gates are small.

`own` false: plain torch operations in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"

FIELDS = dict(op="", f32=False,
              # rotary
              rows=0, heads_q=0, heads_k=0, dim=128, rot=0, axes=1, interleaved=False, inverse=False, table=0, cp=1,
              # norm
              hidden=0, gate="tanh", train=False, unit_offset=False, scale=1.0,
              # attend: samples of `seq` positions of which a cp rank holds 1/cp, and `keys` image tokens each
              batch=1, seq=0, keys=0, img_lo=576, img_hi=576, whole=False,
              # attend_step: requests with len_lo to len_hi encoder states, in a cache with `spare` rows between them
              requests=0, len_lo=0, len_hi=0, spare=0)

MOST_SCORES = 6.6e9          # query heads x rows x keys of a forward pass, which the plain form holds at once
MOST_SCORES_TRAIN = 1.6e9
MOST_ROTARY = 330e6          # values turned
MOST_NORM = 140e6            # values of the residual stream
MOST_BYTES = 2.6e9
MOST_FLOPS = 1.69e12


def _case(name=None, **kw):
    c = dict(FIELDS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decoded token of each of 8 requests: queries and keys turned in one call
        _case("rotary_step", op="rotary", rows=8, heads_q=32, heads_k=8, rot=128, table=32768),
        # one context-parallel rank's rows of a 131072-token sequence, load-balanced split, TP 4 of hidden 5120
        _case("rotary_long", op="rotary", rows=16384, heads_q=10, heads_k=2, rot=128, table=131072, cp=8),
        # a vision encoder's patches: row and column of the grid, heads of 72 channels, binary32, the gradient
        _case("rotary_grid_f32", op="rotary", f32=True, rows=40139, heads_q=16, heads_k=16, dim=72, rot=72, axes=2,
              interleaved=True, inverse=True, table=128),
        # decoding: 8 tokens between two blocks
        _case("norm_step", op="norm", rows=8, hidden=4096),
        # a microbatch of 16384 tokens at hidden 8192, a gate for each channel, forward and backward
        _case("norm_train", op="norm", rows=16384, hidden=8192, gate="channel", train=True, scale=0.5),
        # a hidden size that no vector width divides, binary32, forward and backward
        _case("norm_odd_f32", op="norm", f32=True, rows=4099, hidden=2305, train=True, unit_offset=True),
        # decoding: one request with one image
        _case("attend_step_one", op="attend_step", heads_q=32, heads_k=8, requests=1, len_lo=576, len_hi=576),
        # decoding: 64 requests with 1 to 11 images each, TP 1 of 64 heads
        _case("attend_step_batch", op="attend_step", heads_q=64, heads_k=8, requests=64, len_lo=576, len_hi=6404,
              spare=37),
        # prompts of 4 samples with 7 images each
        _case("attend_prefill", op="attend", batch=4, seq=2048, keys=4032, heads_q=32, heads_k=8, whole=True),
        # one context-parallel rank of the long-context workload: 16384 query rows, 40139 encoder states
        _case("attend_long", op="attend", seq=131072, cp=8, keys=40139, img_lo=256, img_hi=2304, heads_q=10,
              heads_k=2),
        # a training microbatch of TP 2 x CP 2: 8192 query rows, 10 images
        _case("attend_train", op="attend_train", seq=16384, cp=2, keys=5760, heads_q=32, heads_k=4),
        # an encoder's own heads, odd lengths, binary32
        _case("attend_train_f32", op="attend_train", f32=True, batch=3, seq=1025, keys=1153, img_lo=64, img_hi=400,
              heads_q=16, heads_k=16, dim=72),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        if c is None or 3072 in c.values():
            continue
        w = work(c)                                          # no more than the largest listed cases cost
        if w["bytes"] < MOST_BYTES and w["flops"] * (8 if c["f32"] and "attend" in c["op"] else 1) < MOST_FLOPS:
            return c


def _draw(rng):
    op = rng.choice(["rotary", "norm", "attend", "attend_train", "attend_step", "attend_step"])
    f32 = rng.random() < 0.25
    dim = rng.choice([64, 72, 80, 96, 128, 128, 128, 256])
    heads_k = rng.choice([1, 2, 4, 8, 16])
    heads_q = heads_k * rng.choice([1, 1, 2, 3, 4, 5, 8])
    if op == "rotary":
        axes = rng.choice([1, 1, 2, 3])
        rot = rng.choice([dim, dim, dim // 2, dim // 4])
        rows, cp = _log(rng, 1, 131072), rng.choice([1, 2, 4, 8])
        if rows * (heads_q + heads_k) * dim > MOST_ROTARY or (cp > 1 and rows < 2):
            return None
        return _case(op=op, f32=f32, rows=rows, heads_q=heads_q, heads_k=heads_k, dim=dim, rot=rot, axes=axes, cp=cp,
                     interleaved=rng.random() < 0.5, inverse=rng.random() < 0.4,
                     table=min(131072, rows * cp + 512) if axes == 1 else 512)
    if op == "norm":
        kind = rng.random()
        h = _log(rng, 64, 12288)
        hidden = max(1, round(h / 128)) * 128 if kind < 0.55 else max(8, round(h / 8) * 8) if kind < 0.8 else h
        rows = _log(rng, 1, 32768)
        if rows * hidden > MOST_NORM:
            return None
        return _case(op=op, f32=f32, rows=rows, hidden=hidden, gate=rng.choice(["none", "scalar", "tanh", "channel"]),
                     train=rng.random() < 0.5, unit_offset=rng.random() < 0.3, scale=rng.choice([1.0, 0.5]))
    if op == "attend_step":
        lo = _log(rng, 1, 2000)
        hi = _log(rng, lo, 8192)
        requests = _log(rng, 1, 256)
        if requests * requests * (lo + hi) // 2 * heads_q > MOST_SCORES / 4 or heads_q > 64:
            return None
        return _case(op=op, f32=f32, dim=dim, heads_q=heads_q, heads_k=heads_k, requests=requests, len_lo=lo,
                     len_hi=hi, spare=rng.choice([0, 1, 37]))
    cp, batch = rng.choice([1, 1, 2, 8]), rng.choice([1, 1, 2, 5])
    lo = rng.choice([16, 64, 256, 576])
    # with one state to see, the gradients of q and k are zero and a plain form's rounding noise: 16 and more there
    seq, keys = _log(rng, 1, 131072), _log(rng, 16 if op == "attend_train" else 1, 40139)
    seq = max(1, round(seq / (2 * cp))) * 2 * cp if cp > 1 else seq
    most = (MOST_SCORES if op == "attend" else MOST_SCORES_TRAIN) / (8 if f32 else 1)
    scores = batch * (seq // cp) * batch * keys
    if scores * heads_q > most or scores > 7e8 or batch * keys > 80000 or batch * seq // cp * heads_q * dim > 2e8:
        return None
    return _case(op=op, f32=f32, batch=batch, seq=seq, cp=cp, keys=keys, img_lo=lo, img_hi=rng.choice([lo, 4 * lo]),
                 heads_q=heads_q, heads_k=heads_k, dim=dim, whole=rng.random() < 0.3)


# ---- which states a row sees ------------------------------------------------------------------------------

def _ranges(c):
    """(first, end) of the encoder states that each query row sees, and how many states there are.  Belongs to the
    case alone."""
    if c["op"] == "attend_step":
        n = c["requests"]
        lens = [c["len_lo"] + (c["len_hi"] - c["len_lo"]) * (i * 7919 % n) // max(1, n - 1) for i in range(n)]
        starts = np.cumsum([0] + [x + c["spare"] for x in lens])
        return np.stack([starts[:n], starts[:n] + np.array(lens)], 1).astype(np.int32), int(starts[n])
    own_rng = random.Random(c["seq"] * 131 + c["keys"])
    out = []
    for b in range(c["batch"]):
        base = b * c["keys"]
        if c["whole"]:                                   # every row of the sample sees all its states
            rows = np.tile(np.array([[base, base + c["keys"]]]), (c["seq"], 1))
        else:
            lens, left = [], c["keys"]
            while left > 0:
                lens.append(min(left, own_rng.randint(c["img_lo"], c["img_hi"])))
                left -= lens[-1]
            ends = np.sort(np.array([own_rng.randint(0, c["seq"]) for _ in lens]))   # position after each image
            seen = np.concatenate([[0], np.cumsum(lens)])[np.searchsorted(ends, np.arange(c["seq"]), "right")]
            rows = np.stack([np.full(c["seq"], base), base + seen], 1)
        if c["cp"] > 1:                                  # the load-balanced split: the first and the last chunk
            chunk = c["seq"] // (2 * c["cp"])
            rows = np.concatenate([rows[:chunk], rows[-chunk:]])
        out.append(rows)
    return np.concatenate(out).astype(np.int32), c["batch"] * c["keys"]


# ---- inputs ----------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed) + 29)
    dt = torch.float32 if c["f32"] else torch.bfloat16
    new = lambda *shape: torch.randn(shape, generator=g, dtype=dt, device=DEV)  # noqa: E731
    s = {"case": c}
    if c["op"] == "rotary":
        half = c["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        angle = torch.arange(c["table"], dtype=torch.float64, device=DEV)[:, None] * freq
        s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        if c["axes"] == 1:                               # consecutive, or the chunks of a load-balanced split
            p = torch.arange(c["rows"], device=DEV)
            if c["cp"] > 1:
                p = torch.where(p < c["rows"] // 2, p, p + c["rows"] * (c["cp"] - 1))
            if c["rows"] < 512:                          # requests that stand at places of their own
                p = torch.randint(0, c["table"], (c["rows"],), generator=g, device=DEV)
            s["positions"] = (p % c["table"]).to(torch.int32).contiguous()
            s["sections"] = None
        else:                                            # places in a grid
            s["positions"] = torch.randint(0, c["table"], (c["axes"], c["rows"]), generator=g, device=DEV,
                                           dtype=torch.int32)
            each = half // c["axes"]
            s["sections"] = (half - each * (c["axes"] - 1),) + (each,) * (c["axes"] - 1)
        s["x"] = [new(c["rows"], c["heads_q"], c["dim"]), new(c["rows"], c["heads_k"], c["dim"])]
        s["out"] = [torch.empty_like(t) for t in s["x"]]
    elif c["op"] == "norm":
        h = c["hidden"]
        around = 0.0 if c["unit_offset"] else 1.0
        s["x"], s["y"] = new(c["rows"], h), new(c["rows"], h)
        s["w_post"], s["w_pre"] = around + 0.1 * new(h), around + 0.1 * new(h)
        s["gate"] = {"none": None, "scalar": 0.5 * new(1), "tanh": 0.5 * new(1), "channel": 0.3 * new(h)}[c["gate"]]
        s["h"], s["z"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        if c["train"]:
            s["rstd"] = torch.empty(2, c["rows"], dtype=torch.float32, device=DEV)
            s["dh"], s["dz"] = new(c["rows"], h), new(c["rows"], h)
            s["dx"], s["dy"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["dw_post"], s["dw_pre"] = torch.empty_like(s["w_post"]), torch.empty_like(s["w_pre"])
            s["dgate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
    else:
        rng, n_keys = _ranges(c)
        s["ranges"] = torch.from_numpy(rng).to(DEV)
        s["q"] = new(rng.shape[0], c["heads_q"], c["dim"])
        s["k"], s["v"] = new(n_keys, c["heads_k"], c["dim"]), new(n_keys, c["heads_k"], c["dim"])
        s["out"] = torch.empty_like(s["q"])
        if c["op"] == "attend_train":
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
            s["dout"] = new(*s["q"].shape)
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in "qkv")
    return s


# ---- one pass --------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2605_27678_amd as hp
        return {"rotary": _own_rotary, "norm": _own_norm, "attend": _own_attend, "attend_train": _own_attend,
                "attend_step": _own_step}[op](hp, s)
    return {"rotary": _plain_rotary, "norm": _plain_norm, "attend": _plain_attend, "attend_train": _plain_attend,
            "attend_step": _plain_attend}[op](s)


def _workspace(s, size):
    """The scratch memory that a program allocates once for its shapes."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size(), dtype=torch.uint8, device=DEV)
    return s["workspace"]


def _own_rotary(hp, s):
    c = s["case"]
    hp.hp_rotary(s["x"], s["out"], s["table"], s["positions"], interleaved=c["interleaved"], inverse=c["inverse"],
                 sections=s["sections"])
    return s["out"]


def _own_norm(hp, s):
    c = s["case"]
    how = dict(gate_tanh=c["gate"] == "tanh", residual_scale=c["scale"], unit_offset=c["unit_offset"], eps=1e-6)
    if not c["train"]:
        hp.hp_gated_norm(s["x"], s["y"], s["h"], s["z"], s["w_post"], s["gate"], s["w_pre"], **how)
        return {"h": s["h"], "z": s["z"]}
    hp.hp_gated_norm(s["x"], s["y"], s["h"], s["z"], s["w_post"], s["gate"], s["w_pre"], rstd=s["rstd"], **how)
    ws = _workspace(s, lambda: hp.hp_gated_norm_workspace(c["rows"], c["hidden"]))
    hp.hp_gated_norm_backward(s["dh"], s["dz"], s["x"], s["y"], s["rstd"], s["w_post"], s["gate"], s["w_pre"],
                              s["dx"], s["dy"], s["dw_post"], s["dgate"], s["dw_pre"], workspace=ws, **how)
    return {n: s[n] for n in ("h", "z", "dx", "dy", "dw_post", "dgate", "dw_pre")}


def _own_attend(hp, s):
    if s["case"]["op"] == "attend":
        ws = _workspace(s, lambda: hp.hp_cross_attend_workspace(s["q"], s["k"]))
        hp.hp_cross_attend(s["q"], s["k"], s["v"], s["ranges"], s["out"], workspace=ws)
        return s["out"]
    ws = _workspace(s, lambda: max(hp.hp_cross_attend_workspace(s["q"], s["k"]),
                                   hp.hp_cross_attend_workspace(s["q"], s["k"], "backward")))
    hp.hp_cross_attend(s["q"], s["k"], s["v"], s["ranges"], s["out"], lse=s["lse"], workspace=ws)
    hp.hp_cross_attend_backward(s["q"], s["k"], s["v"], s["ranges"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"],
                                s["dv"], workspace=ws)
    return {n: s[n] for n in ("out", "dq", "dk", "dv")}


def _own_step(hp, s):
    ws = _workspace(s, lambda: hp.hp_cross_attend_workspace(s["q"], s["k"], "step"))
    hp.hp_cross_attend_step(s["q"], s["k"], s["v"], s["ranges"], s["out"], workspace=ws)
    return s["out"]


def _plain_rotary(s):
    c = s["case"]
    half = c["rot"] // 2
    if s["sections"] is None:
        turn = s["table"][s["positions"].long()]                                   # [rows, half, 2]
    else:
        axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEV), torch.tensor(s["sections"], device=DEV))
        turn = s["table"][s["positions"].long()[axis].t(), torch.arange(half, device=DEV)]
    cos, sin = turn[:, None, :, 0], turn[:, None, :, 1] * (-1.0 if c["inverse"] else 1.0)
    return [_plain_turn(c, x, cos, sin) for x in s["x"]]


def _plain_turn(c, x, cos, sin):
    f, half = x.float(), c["rot"] // 2
    if c["interleaved"]:
        a, b = f[..., 0:c["rot"]:2], f[..., 1:c["rot"]:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = f[..., :half], f[..., half:c["rot"]]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, f[..., c["rot"]:]], -1).to(x.dtype)


def _plain_norm(s):
    c, eps, dt = s["case"], 1e-6, s["x"].dtype
    x, y = s["x"].float(), s["y"].float()
    w1, w2 = s["w_post"].float(), s["w_pre"].float()
    if c["unit_offset"]:
        w1, w2 = w1 + 1.0, w2 + 1.0
    g = torch.ones(1, device=DEV) if s["gate"] is None else s["gate"].float()
    t = torch.tanh(g) if c["gate"] == "tanh" else g
    r1 = torch.rsqrt(y.square().mean(-1, keepdim=True) + eps)
    n = y * r1 * w1
    h = c["scale"] * x + t * n
    r2 = torch.rsqrt(h.square().mean(-1, keepdim=True) + eps)
    out = {"h": h.to(dt), "z": (h * r2 * w2).to(dt)}
    if not c["train"]:
        return out
    dh, dz = s["dh"].float(), s["dz"].float()
    d = dz * w2
    dh = dh + r2 * d - h * (r2 ** 3 * (h * d).mean(-1, keepdim=True))
    dt_rows = dh * n
    dn = dh * t
    e = dn * w1
    out["dx"] = (c["scale"] * dh).to(dt)
    out["dy"] = (r1 * e - y * (r1 ** 3 * (y * e).mean(-1, keepdim=True))).to(dt)
    out["dw_post"] = (dn * y * r1).sum(0).to(dt)
    out["dw_pre"] = (dz * h * r2).sum(0).to(dt)
    if s["gate"] is None:
        out["dgate"] = None
    elif c["gate"] == "channel":
        out["dgate"] = dt_rows.sum(0).to(dt)
    else:
        out["dgate"] = (dt_rows.sum().reshape(1) * (1.0 - t * t if c["gate"] == "tanh" else 1.0)).to(dt)
    return out


def _by_group(x, heads_k):
    """[rows, heads, dim] -> [heads_k, (heads / heads_k) * rows, dim] in 32 bits."""
    rows, heads, dim = x.shape
    return x.float().permute(1, 0, 2).reshape(heads_k, heads // heads_k * rows, dim)


def _ungroup(x, rows):
    heads_k, m, dim = x.shape
    return x.reshape(heads_k * (m // rows), rows, dim).permute(1, 0, 2)


def _plain_attend(s):
    q, k, v, r = s["q"], s["k"], s["v"], s["ranges"]
    rows, heads_q, dim = q.shape
    n_keys, heads_k = k.shape[:2]
    group, scale, dt = heads_q // heads_k, 1.0 / math.sqrt(dim), q.dtype
    at = torch.arange(n_keys, device=DEV, dtype=torch.int32)
    hidden = (at < r[:, :1]) | (at >= r[:, 1:])                                     # [rows, keys]
    fq, fk, fv = _by_group(q, heads_k), _by_group(k, heads_k), _by_group(v, heads_k)
    p = torch.matmul(fq, fk.transpose(1, 2).contiguous()).mul_(scale)
    p.view(heads_k, group, rows, n_keys).masked_fill_(hidden, float("-inf"))
    top = p.amax(-1, keepdim=True)
    p.sub_(top.masked_fill_(top == float("-inf"), 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total.masked_fill_(total == 0.0, 1.0))
    o = torch.matmul(p, fv)
    out = _ungroup(o, rows).to(dt).contiguous()
    if s["case"]["op"] != "attend_train":
        return out
    do = _by_group(s["dout"], heads_k)
    got = {"out": out, "dv": _ungroup(torch.matmul(p.transpose(1, 2), do), n_keys).to(dt).contiguous()}
    dp = torch.matmul(do, fv.transpose(1, 2).contiguous())
    dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    del p
    got["dq"] = _ungroup(torch.matmul(dp, fk), rows).to(dt).contiguous()
    got["dk"] = _ungroup(torch.matmul(dp.transpose(1, 2), fq), n_keys).to(dt).contiguous()
    return got


# ---- what a pass cannot do without -------------------------------------------------------------------------

def work(case):
    c, e = case, 4 if case["f32"] else 2
    if c["op"] == "rotary":
        values = c["rows"] * (c["heads_q"] + c["heads_k"]) * c["dim"]
        turned = c["rows"] * (c["heads_q"] + c["heads_k"]) * c["rot"]
        return {"bytes": 2 * values * e + c["rows"] * (4 * c["axes"] + 4 * c["rot"]), "flops": 3 * turned}
    if c["op"] == "norm":
        n = c["rows"] * c["hidden"]
        weights = (2 + (c["gate"] == "channel")) * c["hidden"] * e
        if not c["train"]:
            return {"bytes": 4 * n * e + weights, "flops": 11 * n}
        return {"bytes": 10 * n * e + 3 * weights, "flops": 40 * n}
    r, n_keys = _ranges(c)
    pairs = int((r[:, 1].astype(np.int64) - r[:, 0]).sum()) * c["heads_q"]
    q = r.shape[0] * c["heads_q"] * c["dim"] * e
    seen = int((r[:, 1].astype(np.int64) - r[:, 0]).sum()) if c["op"] == "attend_step" else n_keys
    kv = 2 * seen * c["heads_k"] * c["dim"] * e
    if c["op"] == "attend_train":                        # forward: q, k, v -> out; backward: these and dout -> dq, dk, dv
        return {"bytes": 2 * q + kv + (4 * q + 2 * kv), "flops": 14 * pairs * c["dim"]}
    return {"bytes": 2 * q + kv, "flops": 4 * pairs * c["dim"]}


# ---- in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "norm": _exact_norm}.get(case["op"], _exact_attend)(s)


def _exact_rotary(s):
    """Pairs of channels as complex numbers, times the table's."""
    c = s["case"]
    half, table = c["rot"] // 2, torch.view_as_complex(s["table"].double())
    p = s["positions"].long().reshape(c["axes"], c["rows"])
    sections = s["sections"] or (half,)
    begin = [sum(sections[:i]) for i in range(c["axes"])]
    turn = torch.cat([table[p[i]][:, b:b + n] for i, (b, n) in enumerate(zip(begin, sections))], 1)[:, None]
    turn = turn.conj() if c["inverse"] else turn
    out = []
    for x in s["x"]:
        y = x.double().clone()
        first, second = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["interleaved"] else \
            (slice(0, half), slice(half, c["rot"]))
        w = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        y[..., first], y[..., second] = w.real, w.imag
        out.append(y)
    return out


def _exact_norm(s):
    """The definition in 64 bits, its gradients by differentiation of it."""
    c = s["case"]
    leaf = {n: s[n].double().requires_grad_(c["train"]) for n in ("x", "y", "w_post", "w_pre", "gate")
            if s[n] is not None}
    norm = lambda t, w: t / torch.sqrt((t * t).sum(-1, keepdim=True) / c["hidden"] + 1e-6) * (  # noqa: E731
        w + 1 if c["unit_offset"] else w)
    branch = norm(leaf["y"], leaf["w_post"])
    if "gate" in leaf:
        branch = branch * (leaf["gate"].tanh() if c["gate"] == "tanh" else leaf["gate"])
    h = leaf["x"] * c["scale"] + branch
    z = norm(h, leaf["w_pre"])
    out = {"h": h.detach(), "z": z.detach()}
    if c["train"]:
        grads = torch.autograd.grad([h, z], list(leaf.values()), [s["dh"].double(), s["dz"].double()])
        out.update({"d" + n: g for n, g in zip(leaf, grads)})
        out.setdefault("dgate", None)
    return out


def _exact_attend(s):
    """Head by head over the stretch of states that some row sees, or request by request."""
    q, k, v = (s[n].double() for n in "qkv")
    rows, heads_q, dim = q.shape
    n_keys, heads_k = k.shape[:2]
    group = heads_q // heads_k
    lo, hi = s["ranges"].long().unbind(1)
    if s["case"]["op"] == "attend_step":
        out = torch.zeros_like(q)
        for i, (a, b) in enumerate(zip(lo.tolist(), hi.tolist())):
            if b > a:
                score = (q[i].view(heads_k, group, 1, dim) * k[a:b].permute(1, 0, 2)[:, None]).sum(-1) / dim ** 0.5
                w = torch.softmax(score, -1)
                out[i] = (w[..., None] * v[a:b].permute(1, 0, 2)[:, None]).sum(2).reshape(heads_q, dim)
        return out
    train = s["case"]["op"] == "attend_train"
    j = torch.arange(n_keys, device=DEV)
    seen = (j >= lo[:, None]) & (j < hi[:, None])
    some = seen.any(1, keepdim=True)
    out = torch.zeros_like(q)
    grads = {n: torch.zeros_like(t) for n, t in (("dq", q), ("dk", k), ("dv", v))} if train else {}
    for h in range(heads_q):
        a, b, d = (t.contiguous().requires_grad_(train) for t in (q[:, h], k[:, h // group], v[:, h // group]))
        with torch.set_grad_enabled(train):
            score = (a @ b.t().contiguous()) / dim ** 0.5
            score = torch.where(seen, score, torch.full((), -1e300, dtype=torch.float64, device=DEV))
            o = torch.where(some, torch.softmax(score, -1) @ d, torch.zeros((), dtype=torch.float64, device=DEV))
        out[:, h] = o.detach()
        if train:
            da, db, dd = torch.autograd.grad(o, [a, b, d], s["dout"][:, h].double())
            grads["dq"][:, h] = da
            grads["dk"][:, h // group] += db
            grads["dv"][:, h // group] += dd
        del score, o
    return {"out": out, **grads} if train else out
