"""Timed cases of the operators that a mixture-of-experts block needs around its
experts, most of them for training.

Each is given in its plain form (torch, 32 bits; the router's logits and
scores in 64, as they decide whole numbers) and through the package's entry
points:

  norm       the residual stream around a layer: the layer's output normed,
             gated and added to the scaled stream (o), and the norm before the
             next layer (u)
  norm_bwd   its gradients
  route      a router with softmax or sigmoid scores, a bias for balance, groups
             of experts and up to eight experts a token, and the buckets that
             its choices make
  route_bwd  its gradients, the experts' input gradients gathered on the way
  keep8      a matrix to microscaled 8-bit integers (blocks of 32 along the
             rows: int8 values and one power-of-two scale a block) and back
  ffn_train  the experts' FFN forward and backward, its activations kept in
             microscaled 8 bits in between
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_LISTED = [
    # one decoding step at the widest layer's width: latency
    dict(name="norm_token", kind="norm", dtype="bf16", T=1, d=4096, norm="rms", post=True, gate="channel", pre=True),
    # a training batch of the ordinary width, a gate for every token and channel, biases
    dict(name="norm_batch", kind="norm", dtype="bf16", T=8192, d=1024, norm="layer", post=True, gate="token", pre=True),
    # odd sizes in float32: a model small enough to be checked by hand
    dict(name="norm_bwd_odd", kind="norm_bwd", dtype="f32", T=3001, d=1088, norm="layer", post=True, gate="token",
         pre=True),
    # the widest layer's batch
    dict(name="norm_bwd_wide", kind="norm_bwd", dtype="bf16", T=16384, d=4096, norm="rms", post=True, gate="channel",
         pre=True),
    # one token of a decoding stream
    dict(name="route_one", kind="route", dtype="bf16", T=1, d=1024, E=16, k=2, score="softmax", balance=False,
         groups=1, top_groups=1, best=1, renorm=True, cf=0.0),
    # a float32 layer of a few experts, odd token count, capacity
    dict(name="route_odd", kind="route", dtype="f32", T=3001, d=512, E=8, k=3, score="softmax", balance=True,
         groups=1, top_groups=1, best=1, renorm=False, cf=1.1),
    # one GPU's share of an expert-parallel layer's batch: four of eight groups, four experts a token, capacity
    dict(name="route_share", kind="route", dtype="bf16", T=32768, d=2048, E=32, k=4, score="sigmoid", balance=True,
         groups=8, top_groups=4, best=2, renorm=True, cf=1.25),
    # many fine-grained experts, eight a token: the way back of a large batch
    dict(name="route_bwd_many", kind="route_bwd", dtype="bf16", T=65536, d=1024, E=64, k=8, score="sigmoid",
         balance=True, groups=8, top_groups=4, best=2, renorm=True, cf=0.0),
    # a batch's float32 activations of odd row count and a width that is no multiple of 256
    dict(name="keep8_rows", kind="keep8", dtype="f32", rows=3001, cols=1088),
    # the stream of a large batch
    dict(name="keep8_batch", kind="keep8", dtype="bf16", rows=65536, cols=2048),
    # the representatives of 8 x 1024 tokens on the ordinary layer's 16 experts
    dict(name="ffn_ordinary", kind="ffn_train", R=2101, E=16, d=1024, d_ff=4096, act="gelu", zipf=0.0),
    # the representatives of one GPU's share of an expert-parallel layer, Zipf load, some experts nearly idle
    dict(name="ffn_share", kind="ffn_train", R=8653, E=32, d=2048, d_ff=8192, act="silu", zipf=1.1),
]


def listed():
    return [dict(c) for c in _LISTED]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _multiple(v, m):
    return max(m, int(round(v / m)) * m)


def draw(rng):
    """A case of the same ranges: sizes over the logarithm of their range, row
    counts of any parity, widths any multiple of 64 (32 for keep8)."""
    kind = rng.choice(["norm", "norm_bwd", "route", "route", "route_bwd", "keep8", "ffn_train"])
    if kind in ("norm", "norm_bwd"):
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "bf16"]), T=int(_log_uniform(rng, 1, 65536.99)),
                 d=_multiple(_log_uniform(rng, 64, 8192), 64), norm=rng.choice(["rms", "layer"]),
                 post=rng.choice([True, True, False]), gate=rng.choice(["none", "channel", "token"]),
                 pre=rng.choice([True, True, False]))
        while c["T"] * c["d"] > 1 << (24 if c["dtype"] == "f32" else 25):
            c["T"] = c["T"] // 2
        return c
    if kind in ("route", "route_bwd"):
        E = rng.choice([4, 6, 8, 13, 16, 24, 32, 48, 64])
        groups = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0 and E // g >= 2])
        top = rng.randint(max(1, groups // 2), groups)
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "bf16"]), T=int(_log_uniform(rng, 1, 65536.99)),
                 d=_multiple(_log_uniform(rng, 256, 4096), 64), E=E, k=rng.randint(1, min(8, top * (E // groups))),
                 score=rng.choice(["softmax", "sigmoid"]), balance=rng.choice([True, False]), groups=groups,
                 top_groups=top, best=rng.choice([1, 2]), cf=rng.choice([0.0, 1.0, 1.25]))
        c["renorm"] = c["k"] > 1 and rng.choice([True, False])     # one renormalised gate is a constant
        most = (1 << 23) if c["dtype"] == "f32" else (1 << 26)
        if kind == "route_bwd":
            while c["T"] * c["d"] * c["k"] > 1 << 29:
                c["T"] = c["T"] // 2
        while c["T"] * c["d"] > most:
            c["T"] = c["T"] // 2
        return c
    if kind == "keep8":
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), rows=int(_log_uniform(rng, 1, 65536.99)),
                 cols=_multiple(_log_uniform(rng, 32, 11008), 32))
        while c["rows"] * c["cols"] > 1 << (26 if c["dtype"] == "f32" else 27):
            c["rows"] = c["rows"] // 2
        return c
    c = dict(kind=kind, R=int(_log_uniform(rng, 1, 16384.99)), E=rng.choice([4, 6, 8, 13, 16, 24, 32, 48, 64]),
             act=rng.choice(["gelu", "silu"]), zipf=rng.choice([0.0, 0.7, 1.1]))
    c["d"] = _multiple(_log_uniform(rng, 256, 4096), 64)
    c["d_ff"] = _multiple(min(c["d"] * rng.uniform(2.0, 4.0), 11008), 64)
    while 2 * c["E"] * c["d"] * c["d_ff"] > 1 << 30:
        c["E"] = max(4, c["E"] // 2)
        if c["E"] == 4:
            c["d_ff"] = _multiple(c["d_ff"] / 2, 64)
    while c["R"] * c["d"] * c["d_ff"] > 8653 * 2048 * 8192:
        c["R"] = c["R"] // 2
    return c


# ------------------------------------------------------------------ inputs
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-6


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 31)
    return gen


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _weights(gen, shape):
    return torch.randn(shape, generator=gen, dtype=torch.bfloat16, device="cuda").mul_(0.02)


def _activations(gen, rows, cols):
    """Normal rows whose columns differ in size, as hidden states do."""
    spread = torch.exp(0.5 * torch.randn(cols, generator=gen, device="cuda"))
    return torch.randn((rows, cols), generator=gen, device="cuda") * spread


def _counts(case, seed):
    """Rows of every expert: a draw of R rows, some experts possibly without."""
    E = case["E"]
    p = np.arange(1, E + 1, dtype=np.float64) ** (-case["zipf"])
    rng = np.random.RandomState((int(seed) * 7919 + 17) % (1 << 32))
    return rng.multinomial(case["R"], rng.permutation(p / p.sum()))


def _prepare_norm(case, gen):
    dt, T, d = _TYPES[case["dtype"]], case["T"], case["d"]
    s = dict(kind=case["kind"], norm=case["norm"], dt=dt, alpha=0.9, post=case["post"], pre=case["pre"], wp=None,
             bp=None, g=None, w=None, b=None)
    layer = case["norm"] == "layer"
    if case["post"]:
        s["wp"] = 1.0 + 0.1 * _randn(gen, d)
        s["bp"] = 0.1 * _randn(gen, d) if layer else None
    if case["gate"] == "channel":
        s["g"] = 0.5 + 0.1 * _randn(gen, d)
    elif case["gate"] == "token":
        s["g"] = torch.sigmoid(_randn(gen, T, d)).to(dt)
    if case["pre"]:
        s["w"] = 1.0 + 0.1 * _randn(gen, d)
        s["b"] = 0.1 * _randn(gen, d) if layer else None
    s["y"] = (0.3 * _activations(gen, T, d) + 0.05).to(dt)
    if case["kind"] == "norm":
        s["x"] = _activations(gen, T, d).to(dt)
    else:
        s["o"] = (_activations(gen, T, d) + 0.1).to(dt)
        s["do"] = _randn(gen, T, d).to(dt)
        s["du"] = _randn(gen, T, d).to(dt) if case["pre"] else None
    return s


def _prepare_route(case, gen):
    dt, T, d, E, k = _TYPES[case["dtype"]], case["T"], case["d"], case["E"], case["k"]
    s = {n: case[n] for n in ("kind", "k", "score", "groups", "top_groups", "best", "renorm", "cf")}
    s.update(dt=dt, scale=1.0 if case["score"] == "softmax" else 2.5)
    s["x"] = _activations(gen, T, d).to(dt)
    s["w"] = (0.02 * _randn(gen, E, d)).to(dt)
    s["b"] = 0.1 * _randn(gen, E)
    s["balance"] = (0.05 if case["score"] == "sigmoid" else 0.5 / E) * _randn(gen, E) if case["balance"] else None
    if case["kind"] == "route_bwd":      # what the way there and the experts have left
        f = _plain_route(s)
        s.update(logits=f["logits"], idx=f["idx"], slot_pos=f["slot_pos"])
        S = int(f["offsets"][-1])
        rep = torch.rand(T * k, generator=gen, device="cuda") < 0.6
        rep[f["offsets"][:-1].long().clamp_max(T * k - 1)] = True
        own_place = torch.where(rep, torch.arange(T * k, device="cuda"), -1)
        s["rep_of_pos"] = torch.cummax(own_place, 0).values.clamp_min(0).to(torch.int32)
        s["rep_row"] = (torch.cumsum(rep[:S], 0) - 1)[s["rep_of_pos"][:S].long()].to(torch.int32)
        s["rep_row"] = torch.nn.functional.pad(s["rep_row"], (0, T * k - S))
        s["dgate"] = torch.where(s["slot_pos"] >= 0, _randn(gen, T, k), torch.zeros((), device="cuda"))
        s["dx_rep"] = torch.randn((T * k, d), generator=gen, dtype=torch.bfloat16, device="cuda").to(dt)
    return s


def _prepare_ffn(case, seed, gen):
    E, d, d_ff, R = case["E"], case["d"], case["d_ff"], case["R"]
    n = _counts(case, seed)
    tokens = max(1, (R * 3) // 2)
    return dict(kind=case["kind"], act=case["act"], R=R, most=max(1, int(n.max())),
                x=_activations(gen, tokens, d).to(torch.bfloat16),
                index=torch.randint(0, tokens, (R,), generator=gen, device="cuda").to(torch.int32),
                offsets=torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda(),
                w1=_weights(gen, (E, d_ff, d)), w2=_weights(gen, (E, d, d_ff)),
                dy=_randn(gen, R, d).to(torch.bfloat16))


def prepare(case, seed):
    """Inputs, and the weights as the program keeps them."""
    gen = _generator(seed)
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        return _prepare_norm(case, gen)
    if kind in ("route", "route_bwd"):
        return _prepare_route(case, gen)
    if kind == "keep8":
        return dict(kind=kind, x=_activations(gen, case["rows"], case["cols"]).to(_TYPES[case["dtype"]]))
    return _prepare_ffn(case, seed, gen)


# ------------------------------------------------------------- plain forms
def _normed(a, norm):
    """(a - mean) r and r of the rows of a (float32)."""
    if norm == "layer":
        a = a - a.mean(1, keepdim=True)
    r = torch.rsqrt((a * a).mean(1, keepdim=True) + _EPS)
    return a * r, r


def _plain_norm(s):
    v = s["y"].float()
    if s["post"]:
        v = _normed(v, s["norm"])[0] * s["wp"]
        if s["bp"] is not None:
            v = v + s["bp"]
    if s["g"] is not None:
        v = v * s["g"].float()
    o = (s["alpha"] * s["x"].float() + v).to(s["dt"])
    out = dict(o=o)
    if s["pre"]:                         # of the stream as it is stored
        u = _normed(o.float(), s["norm"])[0] * s["w"]
        out["u"] = (u if s["b"] is None else u + s["b"]).to(s["dt"])
    return out


def _normed_back(q, ahat, r, norm):
    """Gradient of the rows a from that of their normed form."""
    p = q - ahat * (q * ahat).mean(1, keepdim=True)
    return r * (p - q.mean(1, keepdim=True) if norm == "layer" else p)


def _plain_norm_bwd(s):
    out = {}
    do = s["do"].float()
    if s["pre"]:
        ohat, r = _normed(s["o"].float(), s["norm"])
        du = s["du"].float()
        out["dw"] = (du * ohat).sum(0)
        if s["b"] is not None:
            out["db"] = du.sum(0)
        do = do + _normed_back(du * s["w"], ohat, r, s["norm"])
    out["dx"] = (s["alpha"] * do).to(s["dt"])
    v = y = s["y"].float()
    if s["post"]:
        yhat, r = _normed(y, s["norm"])
        v = yhat * s["wp"]
        if s["bp"] is not None:
            v = v + s["bp"]
    dv = do
    if s["g"] is not None:
        dv = do * s["g"].float()
        dg = do * v
        out["dg"] = dg.sum(0) if s["g"].dim() == 1 else dg.to(s["dt"])
    if s["post"]:
        out["dwp"] = (dv * yhat).sum(0)
        if s["bp"] is not None:
            out["dbp"] = dv.sum(0)
        dv = _normed_back(dv * s["wp"], yhat, r, s["norm"])
    out["dy"] = dv.to(s["dt"])
    return out


def _choose(c, rank, s):
    """The k largest of rank [T, E] in the groups with the best c, the lower
    index first among equal ones."""
    T, E = c.shape
    if s["top_groups"] < s["groups"]:
        size = E // s["groups"]
        best = torch.sort(c.view(T, s["groups"], size), dim=2, descending=True).values[..., : min(s["best"], size)]
        order = torch.sort(best.sum(2), dim=1, descending=True, stable=True).indices[:, : s["top_groups"]]
        kept = torch.zeros(T, s["groups"], dtype=torch.bool, device=c.device).scatter_(1, order, True)
        rank = torch.where(kept.repeat_interleave(size, dim=1), rank, torch.full_like(rank, -math.inf))
    return torch.sort(rank, dim=1, descending=True, stable=True).indices[:, : s["k"]]


def _scores(l, score):
    return torch.softmax(l, 1) if score == "softmax" else 1.0 / (1.0 + torch.exp(-l))


def _plain_route(s):
    T, E, k = s["x"].shape[0], s["w"].shape[0], s["k"]
    l = torch.matmul(s["x"].double(), s["w"].double().t()) + s["b"].double()
    sc = _scores(l, s["score"])
    if s["balance"] is not None:
        c = rank = sc + s["balance"].double()
    else:                                # in the order of the logits: scores may be equal where they are not
        c, rank = (l if s["best"] == 1 else sc), l
    idx = _choose(c, rank, s)
    g = sc.gather(1, idx)
    if s["renorm"]:
        g = g / g.sum(1, keepdim=True)
    # buckets: slots in the order of their choice, then of their token
    flat = idx.t().reshape(-1)
    order = torch.sort(flat, stable=True).indices
    n = torch.bincount(flat, minlength=E)
    start = torch.cumsum(n, 0) - n
    place = torch.empty_like(flat)
    place[order] = torch.arange(T * k, device=flat.device) - start[flat[order]]
    kept_n = n
    if s["cf"] > 0:
        kept_n = n.clamp_max(math.ceil(s["cf"] * k * T / E - 1e-9))
    offsets = torch.nn.functional.pad(torch.cumsum(kept_n, 0), (1, 0))
    pos = torch.where(place < kept_n[flat], offsets[flat] + place, torch.full_like(place, -1))
    perm = torch.zeros(T * k + 1, dtype=torch.int64, device=flat.device)
    perm[torch.where(pos >= 0, pos, torch.full_like(pos, T * k))] = torch.arange(T, device=flat.device).repeat(k)
    i32 = torch.int32
    return dict(idx=idx.to(i32), gate=(g * s["scale"]).float(), logits=l.float(),
                slot_pos=pos.view(k, T).t().to(i32).contiguous(), perm_token=perm[:-1].to(i32),
                offsets=offsets.to(i32))


def _plain_route_bwd(s):
    l, idx, dgate = s["logits"], s["idx"].long(), s["dgate"]
    sc = _scores(l, s["score"])
    g = sc.gather(1, idx)
    if s["renorm"]:
        n = g.sum(1, keepdim=True)
        ds = s["scale"] / n * (dgate - (dgate * g).sum(1, keepdim=True) / n)
    else:
        ds = s["scale"] * dgate
    ds = torch.zeros_like(sc).scatter_(1, idx, ds)
    if s["score"] == "softmax":
        dl = sc * (ds - (ds * sc).sum(1, keepdim=True))
    else:
        dl = ds * sc / (1.0 + torch.exp(l))
    x = s["x"].float()
    dx = torch.matmul(dl, s["w"].float())
    p = s["slot_pos"].long()
    held = p.clamp_min(0)
    mine = (p >= 0) & (s["rep_of_pos"][held] == s["slot_pos"])
    row = torch.where(mine, s["rep_row"][held].long(), torch.zeros_like(held))
    dx = dx + torch.where(mine[..., None], s["dx_rep"][row].float(), torch.zeros((), device=x.device)).sum(1)
    return dict(dx=dx.to(s["dt"]), dw=torch.matmul(dl.t(), x), db=dl.sum(0))


def _power_of_two(n):
    """2^n, -126 <= n <= 127, exactly (pow need not be)."""
    return ((n + 127) << 23).view(torch.float32)


def _round8(v):
    """v [.., K] (float32) to microscaled 8-bit integers and back."""
    b = v.reshape(*v.shape[:-1], -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    scale = torch.clamp(torch.frexp(most).exponent.to(torch.int32) - 1 - 6, min=-127)
    scale = torch.where(most == 0, torch.full_like(scale, -127), scale)
    # in two steps: 2^127 and 2^-127 stay in range
    half = scale >> 1
    u = torch.clamp(torch.round(b * _power_of_two(-half) * _power_of_two(half - scale)), -127.0, 127.0)
    return (u * _power_of_two(half) * _power_of_two(scale - half)).reshape(v.shape)


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z / (1.0 + torch.exp(-z))


def _act_slope(z, act):
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    q = 1.0 / (1.0 + torch.exp(-z))
    return q * (1.0 + z * (1.0 - q))


def _plain_ffn(s):
    off, R, act, bf = s["offsets"].long(), s["R"], s["act"], torch.bfloat16
    at = off[:-1, None] + torch.arange(s["most"], device=off.device)
    used = at < off[1:, None]
    rows = torch.minimum(at, off[1:, None] - 1).clamp_(0, R - 1)              # [E, most]
    w1, w2 = s["w1"].float(), s["w2"].float()
    x = s["x"].float()
    index = s["index"].long()[rows]
    z = torch.matmul(x[index], w1.transpose(1, 2))
    y = torch.matmul(_act(z, act), w2.transpose(1, 2))[used]
    z = _round8(z)                                                            # what is kept of it
    dy = torch.where(used[..., None], s["dy"].float()[rows], torch.zeros((), device=x.device))
    dw2 = torch.matmul(dy.transpose(1, 2), _act(z, act))
    dz = torch.matmul(dy, w2) * _act_slope(z, act)
    dw1 = torch.matmul(dz.transpose(1, 2), _round8(x)[index])
    dx = torch.matmul(dz, w1)[used]
    return dict(y=y.to(bf), dx=dx.to(bf), dw1=dw1.to(bf), dw2=dw2.to(bf))


# -------------------------------------------------- the package's operators
def _buffer(s, name, shape, dtype):
    """An output or workspace that the program keeps from step to step."""
    if name not in s:
        s[name] = torch.zeros(shape, dtype=dtype, device="cuda")
    return s[name]


def _own_norm(s):
    import paper_2411_15419_amd as luffy
    o = _buffer(s, "o", s["x"].shape, s["dt"])
    u = _buffer(s, "u", s["x"].shape, s["dt"]) if s["pre"] else None
    luffy.luffy_block_norm(s["x"], s["y"], o, u, norm=s["norm"], eps=_EPS, res_scale=s["alpha"], w_post=s["wp"],
                           b_post=s["bp"], gate=s["g"], w_pre=s["w"], b_pre=s["b"])
    return dict(o=o) if u is None else dict(o=o, u=u)


def _own_norm_bwd(s):
    import paper_2411_15419_amd as luffy
    T, d = s["y"].shape
    f32, g = torch.float32, s["g"]
    out = dict(dx=_buffer(s, "dx", (T, d), s["dt"]), dy=_buffer(s, "dy", (T, d), s["dt"]))
    if g is not None:
        out["dg"] = _buffer(s, "dg", g.shape, g.dtype)
    for name, of in (("dw", "w"), ("db", "b"), ("dwp", "wp"), ("dbp", "bp")):
        if s[of] is not None:
            out[name] = _buffer(s, name, (d,), f32)
    ws = _buffer(s, "workspace", luffy.block_norm_backward_workspace_size(T, d), torch.uint8)
    luffy.luffy_block_norm_backward(s["y"], s["o"], s["do"], s["du"], out["dx"], out["dy"], ws, norm=s["norm"],
                                    eps=_EPS, res_scale=s["alpha"], w_post=s["wp"], b_post=s["bp"], gate=g,
                                    w_pre=s["w"], dgate=out.get("dg"), dw_post=out.get("dwp"),
                                    db_post=out.get("dbp"), dw_pre=out.get("dw"), db_pre=out.get("db"))
    return out


def _own_route(s):
    import paper_2411_15419_amd as luffy
    T, E, k = s["x"].shape[0], s["w"].shape[0], s["k"]
    i32, f32 = torch.int32, torch.float32
    out = dict(idx=_buffer(s, "idx", (T, k), i32), gate=_buffer(s, "gate", (T, k), f32),
               logits=_buffer(s, "logits", (T, E), f32), slot_pos=_buffer(s, "slot_pos", (T, k), i32),
               perm_token=_buffer(s, "perm_token", (T * k,), i32), offsets=_buffer(s, "offsets", (E + 1,), i32))
    ws = _buffer(s, "workspace", luffy.route_workspace_size(T, E, k), torch.uint8)
    luffy.luffy_route_scored(s["x"], s["w"], s["b"], k, s["score"], s["cf"], out["idx"], out["gate"], out["logits"],
                             out["slot_pos"], out["perm_token"], out["offsets"], ws, balance=s["balance"],
                             groups=s["groups"], top_groups=s["top_groups"], group_best=s["best"],
                             renormalise=s["renorm"], scale=s["scale"])
    return out


def _own_route_bwd(s):
    import paper_2411_15419_amd as luffy
    T, d = s["x"].shape
    E = s["w"].shape[0]
    out = dict(dx=_buffer(s, "dx", (T, d), s["dt"]), dw=_buffer(s, "dw", (E, d), torch.float32),
               db=_buffer(s, "db", (E,), torch.float32))
    ws = _buffer(s, "workspace", luffy.route_scored_backward_workspace_size(T, d, E), torch.uint8)
    luffy.luffy_route_scored_backward(s["x"], s["w"], s["score"], s["logits"], s["idx"], s["dgate"], out["dx"],
                                      out["dw"], out["db"], ws, renormalise=s["renorm"], scale=s["scale"],
                                      dx_rep=s["dx_rep"], slot_pos=s["slot_pos"], rep_of_pos=s["rep_of_pos"],
                                      rep_row=s["rep_row"])
    return out


def _kept8(s, name, rows, cols):
    return (_buffer(s, name + "_q", (rows, cols), torch.int8),
            _buffer(s, name + "_s", ((cols + 255) // 256, rows, 8), torch.uint8))


def _own_keep8(s):
    import paper_2411_15419_amd as luffy
    x = s["x"]
    q, sc = _kept8(s, "x", *x.shape)
    y = _buffer(s, "y", x.shape, x.dtype)
    luffy.luffy_mx8_quantize(x, q, sc)
    luffy.luffy_mx8_dequantize(q, sc, y)
    return y


def _own_ffn(s):
    import paper_2411_15419_amd as luffy
    R, x, bf = s["R"], s["x"], torch.bfloat16
    E, d_ff, d = s["w1"].shape
    xq, xs = _kept8(s, "x", *x.shape)
    zq, zs = _kept8(s, "z", R, d_ff)
    out = dict(y=_buffer(s, "y", (R, d), bf), dx=_buffer(s, "dx", (R, d), bf),
               dw1=_buffer(s, "dw1", s["w1"].shape, bf), dw2=_buffer(s, "dw2", s["w2"].shape, bf))
    ws = _buffer(s, "workspace", luffy.expert_ffn_workspace_size(R, E, d_ff, luffy.LUFFY_BF16), torch.uint8)
    ws_b = _buffer(s, "workspace_b", luffy.expert_ffn_backward_kept_workspace_size(R, E, d, d_ff), torch.uint8)
    luffy.luffy_mx8_quantize(x, xq, xs)
    luffy.luffy_expert_ffn_keep(x, s["index"], s["offsets"], s["w1"], s["w2"], s["act"], R, zq, zs, out["y"], ws)
    luffy.luffy_expert_ffn_backward_kept(xq, xs, s["index"], s["offsets"], s["w1"], s["w2"], s["act"], R, zq, zs,
                                         s["dy"], out["dx"], out["dw1"], out["dw2"], ws_b)
    return out


def run(state):
    """One pass: a block's norms, a router, rows to 8 bits and back, or the
    experts' training step."""
    kind = state["kind"]
    if own:
        return dict(norm=_own_norm, norm_bwd=_own_norm_bwd, route=_own_route, route_bwd=_own_route_bwd,
                    keep8=_own_keep8, ffn_train=_own_ffn)[kind](state)
    if kind == "keep8":
        return _round8(state["x"].float()).to(state["x"].dtype)
    return dict(norm=_plain_norm, norm_bwd=_plain_norm_bwd, route=_plain_route, route_bwd=_plain_route_bwd,
                ffn_train=_plain_ffn)[kind](state)


# -------------------------------------------------------------------- work
def work(case):
    """Bytes: inputs and the weights of the experts in use read once, outputs
    written once (keep8: also its 8-bit form, written and read back; ffn_train:
    the kept activations too, the gathered rows once each way).  Flops: the
    products."""
    kind = case["kind"]
    if kind == "keep8":
        n = float(case["rows"]) * case["cols"]
        return {"bytes": n * 2 * (4 if case["dtype"] == "f32" else 2) + 2 * n * (1 + 1 / 32), "flops": 0.0}
    if kind == "ffn_train":
        R, d, d_ff = float(case["R"]), case["d"], case["d_ff"]
        used = float((_counts(case, 0) > 0).sum())
        weights = 2 * used * d * d_ff * 2 * 2 + 2 * case["E"] * d * d_ff * 2.0     # read twice, gradients written
        kept = 2 * R * (d + d_ff) * (1 + 1 / 32)
        return {"bytes": weights + kept + R * d * 2 * 4, "flops": 6 * 2 * R * d * d_ff}
    T, d = float(case["T"]), case["d"]
    b = 4 if case["dtype"] == "f32" else 2
    if kind in ("norm", "norm_bwd"):
        n = 3 + case["pre"] if kind == "norm" else 4 + 2 * case["pre"]   # x y o (u); y do dx dy (o du)
        if case["gate"] == "token":
            n += 1 if kind == "norm" else 2
        vectors = 4.0 * d * ((1 + (case["norm"] == "layer")) * (case["post"] + case["pre"]) + (case["gate"] == "channel"))
        return {"bytes": n * T * d * b + vectors * (1 if kind == "norm" else 2), "flops": 0.0}
    E, k = case["E"], case["k"]
    if kind == "route":
        return {"bytes": T * d * b + E * d * b + 4 * T * E + 16 * T * k, "flops": 2 * T * d * E}
    kept = min(1.0, case["cf"]) if case["cf"] else 1.0                 # about: of the slots that are in a bucket
    return {"bytes": 2 * T * d * b + E * d * (b + 4) + 4 * T * E + 0.6 * kept * T * k * d * b + 20 * T * k,
            "flops": 4 * T * d * E}


# ------------------------------------------------------------------- exact
def _exact_norm(s):
    def n64(a, w, bias):
        a = a.double()
        mean = a.sum(1) / a.shape[1] if s["norm"] == "layer" else torch.zeros_like(a[:, 0])
        dev = a - mean[:, None]
        a = dev / torch.sqrt((dev ** 2).sum(1) / a.shape[1] + _EPS)[:, None] * w.double()
        return a if bias is None else a + bias.double()

    v = n64(s["y"], s["wp"], s["bp"]) if s["post"] else s["y"].double()
    g = 1.0 if s["g"] is None else s["g"].double()
    o = s["alpha"] * s["x"].double() + g * v
    out = dict(o=o)
    if s["pre"]:
        out["u"] = n64(o.to(s["dt"]), s["w"], s["b"])
    return out


def _exact_norm_bwd(s):
    """By automatic differentiation of the definition, in 64 bits."""
    names = [n for n in ("wp", "bp", "g", "w", "b") if s[n] is not None]
    p = {n: s[n].double().requires_grad_() for n in names}
    y = s["y"].double().requires_grad_()
    r = s["o"].double().requires_grad_()     # the stream where it is read

    def n64(a, w, bias):
        if s["norm"] == "layer":
            a = a - a.mean(1, keepdim=True)
        a = a / torch.sqrt(a.square().mean(1, keepdim=True) + _EPS) * w
        return a if bias is None else a + bias

    out = {}
    total = s["do"].double()
    if s["pre"]:
        wanted = [r] + [p[n] for n in ("w", "b") if n in p]
        got = torch.autograd.grad(n64(r, p["w"], p.get("b")), wanted, s["du"].double())
        total = total + got[0]
        out.update(zip(["d" + n for n in ("w", "b") if n in p], got[1:]))
    v = n64(y, p["wp"], p.get("bp")) if s["post"] else y * 1.0
    v = v * p["g"] if "g" in p else v
    rest = [n for n in ("wp", "bp", "g") if n in p]
    got = torch.autograd.grad(v, [y] + [p[n] for n in rest], total)
    out.update(dx=s["alpha"] * total, dy=got[0])
    out.update(zip(["d" + n for n in rest], got[1:]))
    return out


def _exact_route(s):
    f = _plain_route(s)                      # whole numbers: which experts
    l = s["x"].double() @ s["w"].double().t() + s["b"].double()
    chosen = l.gather(1, f["idx"].long())
    if s["score"] == "softmax":
        g = torch.softmax(chosen, 1) if s["renorm"] else torch.exp(chosen - torch.logsumexp(l, 1, keepdim=True))
    else:
        g = torch.sigmoid(chosen)
        g = g / g.sum(1, keepdim=True) if s["renorm"] else g
    return dict(idx=None, gate=g * s["scale"], logits=l, slot_pos=None, perm_token=None, offsets=None)


def _exact_route_bwd(s):
    l = s["logits"].double().requires_grad_()
    idx = s["idx"].long()
    sc = torch.softmax(l, 1) if s["score"] == "softmax" else torch.sigmoid(l)
    g = sc.gather(1, idx)
    g = g / g.sum(1, keepdim=True) if s["renorm"] else g
    dl, = torch.autograd.grad(g * s["scale"], l, s["dgate"].double())
    dx = dl @ s["w"].double()
    T, k = idx.shape
    for j in range(k):
        t = torch.arange(T, device=l.device)
        p = s["slot_pos"][:, j].long()
        t, p = t[p >= 0], p[p >= 0]
        mine = s["rep_of_pos"][p].long() == p
        dx.index_add_(0, t[mine], s["dx_rep"][s["rep_row"][p[mine]].long()].double())
    return dict(dx=dx, dw=dl.t() @ s["x"].double(), db=dl.sum(0))


def _round64(v):
    """v to microscaled 8-bit integers and back, in 64 bits."""
    b = v.double().reshape(v.shape[0], -1, 32)
    most = b.abs().amax(2, keepdim=True)
    e = torch.where(most > 0, (most.view(torch.int64) >> 52) - 1023, -127 + 6)    # the exponent's field
    step = ((torch.clamp(e - 6, min=-127) + 1023) << 52).view(torch.float64)
    return (torch.clamp(torch.round(b / step), -127, 127) * step).reshape(v.shape)


def _exact_ffn(s):
    off = s["offsets"].tolist()
    d = s["x"].shape[1]
    y, dx = (torch.zeros((s["R"], d), dtype=torch.float64, device="cuda") for _ in range(2))
    dw1, dw2 = (torch.zeros(s[n].shape, dtype=torch.float32, device="cuda") for n in ("w1", "w2"))
    for e in range(len(off) - 1):
        a, b = off[e], off[e + 1]
        if b > a:
            index = s["index"][a:b].long()
            w1, w2, dy = s["w1"][e].double(), s["w2"][e].double(), s["dy"][a:b].double()
            z = s["x"][index].double() @ w1.t()
            gelu = s["act"] == "gelu"
            y[a:b] = (z * (torch.special.ndtr(z) if gelu else torch.sigmoid(z))) @ w2.t()
            z = _round64(z)
            q = torch.special.ndtr(z) if gelu else torch.sigmoid(z)
            slope = q + z * (torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if gelu else q * (1 - q))
            dz = (dy @ w2) * slope
            dx[a:b] = dz @ w1
            dw1[e] = dz.t() @ _round64(s["x"][index])
            dw2[e] = dy.t() @ (z * q)
    return dict(y=y, dx=dx, dw1=dw1, dw2=dw2)


def exact(case, seed):
    """run()'s floating outputs from the operators' definitions in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] == "keep8":
        return _round64(s["x"])
    return dict(norm=_exact_norm, norm_bwd=_exact_norm_bwd, route=_exact_route, route_bwd=_exact_route_bwd,
                ffn_train=_exact_ffn)[case["kind"]](s)
