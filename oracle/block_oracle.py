"""Plain 64-bit forms of the operators around and inside a training block: the
norms with gate and residual, the scored router, activations kept in
microscaled 8 bits and the experts' FFN on them, each with its gradients.
Written from the definitions in include/luffy.h; numpy only."""
from __future__ import annotations

import math

import numpy as np

from .luffy_oracle import activation, activation_grad, capacity_of


# ------------------------------------------------------------------ norms
def norm_rows(a, norm, eps):
    """(a - m) r and r of every row."""
    a = np.asarray(a, np.float64)
    if norm == "layer":
        a = a - a.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((a * a).mean(1, keepdims=True) + eps)
    return a * r, r


def block_norm(x, y, *, norm, eps, res_scale=1.0, w_post=None, b_post=None, gate=None):
    """o of the stream x and a layer's output y."""
    v = np.asarray(y, np.float64)
    if w_post is not None:
        v = norm_rows(v, norm, eps)[0] * w_post + (0.0 if b_post is None else b_post)
    return res_scale * np.asarray(x, np.float64) + (1.0 if gate is None else gate) * v


def pre_norm(o, *, norm, eps, w_pre, b_pre=None):
    return norm_rows(o, norm, eps)[0] * w_pre + (0.0 if b_pre is None else b_pre)


def _through(q, ahat, r, norm):
    """Gradient of the rows from q, that of their normed form."""
    p = q - ahat * (q * ahat).mean(1, keepdims=True)
    return r * (p - q.mean(1, keepdims=True) if norm == "layer" else p)


def block_norm_backward(y, o, dout, du, *, norm, eps, res_scale=1.0, w_post=None, b_post=None, gate=None, w_pre=None):
    """Gradients (a dict; a channel gate's and the weights' summed over rows)."""
    out = {}
    total = 0.0 if dout is None else np.asarray(dout, np.float64)
    if du is not None:
        ohat, r = norm_rows(o, norm, eps)
        out["dw_pre"], out["db_pre"] = (du * ohat).sum(0), np.asarray(du, np.float64).sum(0)
        total = total + _through(du * w_pre, ohat, r, norm)
    out["dx"] = res_scale * total
    if y is None:
        return out
    v = np.asarray(y, np.float64)
    if w_post is not None:
        yhat, r = norm_rows(y, norm, eps)
        v = yhat * w_post + (0.0 if b_post is None else b_post)
    dv = total
    if gate is not None:
        out["dgate"] = (total * v).sum(0) if np.ndim(gate) == 1 else total * v
        dv = total * gate
    if w_post is not None:
        out["dw_post"], out["db_post"] = (dv * yhat).sum(0), dv.sum(0)
        dv = _through(dv * w_post, yhat, r, norm)
    out["dy"] = dv
    return out


# ----------------------------------------------------------------- router
def scores(l, score):
    if score == "sigmoid":
        return 1.0 / (1.0 + np.exp(-l))
    e = np.exp(l - l.max(1, keepdims=True))
    return e / e.sum(1, keepdims=True)


def choose(l, k, score, balance=None, groups=1, top_groups=1, group_best=1):
    """The chosen experts [T, k], best first, the lower index first among equal
    ones.  One token and one comparison at a time."""
    T, E = l.shape
    s = scores(l, score)
    c = l if balance is None else s + balance
    gc = s if balance is None and group_best == 2 else c
    size = E // groups
    idx = np.zeros((T, k), np.int64)
    for t in range(T):
        kept = list(range(groups))
        if top_groups < groups:
            value = [sum(sorted(gc[t, g * size:(g + 1) * size])[::-1][:group_best]) for g in range(groups)]
            kept = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
        allowed = sorted(e for g in kept for e in range(g * size, (g + 1) * size))
        idx[t] = sorted(allowed, key=lambda e: (-c[t, e], e))[:k]
    return idx


def gates(l, idx, score, renormalise, scale=1.0):
    g = np.take_along_axis(scores(l, score), idx, 1)
    return scale * (g / g.sum(1, keepdims=True) if renormalise else g)


def buckets(idx, E, capacity_factor=0.0):
    """(slot_pos [T, k], perm_token, offsets): slots s = j T + t in order, the
    first C of every expert."""
    T, k = idx.shape
    C = capacity_of(T, k, E, capacity_factor)
    lists = [[] for _ in range(E)]
    place = {}
    for j in range(k):
        for t in range(T):
            e = idx[t, j]
            if C <= 0 or len(lists[e]) < C:
                place[t, j] = (e, len(lists[e]))
                lists[e].append(t)
    offsets = np.concatenate([[0], np.cumsum([len(b) for b in lists])])
    slot_pos = np.full((T, k), -1, np.int64)
    for (t, j), (e, p) in place.items():
        slot_pos[t, j] = offsets[e] + p
    return slot_pos, np.array([t for b in lists for t in b], np.int64), offsets


def dlogits(l, idx, dgate, score, renormalise, scale=1.0):
    """Gradient in the logits of sum(dgate * gates)."""
    s = scores(l, score)
    g = np.take_along_axis(s, idx, 1)
    if renormalise:
        n = g.sum(1, keepdims=True)
        ds_chosen = scale * (dgate / n - (dgate * g).sum(1, keepdims=True) / n ** 2)
    else:
        ds_chosen = scale * dgate
    ds = np.zeros_like(s)
    np.put_along_axis(ds, idx, ds_chosen, 1)
    if score == "sigmoid":
        return ds * s * (1.0 / (1.0 + np.exp(l)))
    return s * (ds - (ds * s).sum(1, keepdims=True))


def route_backward(x, w, l, idx, dgate, score, renormalise, scale=1.0, extra=None, dx_rep=None, slot_pos=None,
                   rep_of_pos=None, rep_row=None):
    """(dx, dw, db)."""
    dl = dlogits(l, idx, dgate, score, renormalise, scale) + (0.0 if extra is None else extra)
    dx = dl @ np.asarray(w, np.float64)
    if dx_rep is not None:
        for t in range(idx.shape[0]):
            for p in slot_pos[t]:
                if p >= 0 and rep_of_pos[p] == p:
                    dx[t] += dx_rep[rep_row[p]]
    return dx, dl.T @ np.asarray(x, np.float64), dl.sum(0)


# ------------------------------------------------- microscaled 8-bit integers
def mx8_quantize(x):
    """x [rows, cols] -> int8 [rows, cols], scale bytes [rows, cols/32]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    b = x.reshape(rows, cols // 32, 32)
    finite = np.isfinite(b).all(-1)
    b = np.where(finite[..., None], b, 0.0)
    most = np.abs(b).max(-1)
    e = np.where(most > 0, np.maximum(np.frexp(most)[1] - 1 - 6, -127), -127)
    q = np.clip(np.rint(np.ldexp(b, -e[..., None])), -127, 127).astype(np.int8)
    return q.reshape(rows, cols), np.where(finite, e + 127, 255).astype(np.uint8)


def mx8_values(q, s):
    f = np.where(s == 255, np.nan, np.ldexp(1.0, s.astype(np.int64) - 127))
    return q.astype(np.float64) * np.repeat(f, 32, axis=-1)


def mx8_rounded(x):
    return mx8_values(*mx8_quantize(x))


def pack_scales(s):
    """Scale bytes [rows, n] as stored: [ceil(n/8), rows, 8]."""
    rows, n = s.shape
    p = np.zeros((rows, (n + 7) // 8 * 8), np.uint8)
    p[:, :n] = s
    return np.ascontiguousarray(p.reshape(rows, -1, 8).transpose(1, 0, 2))


def unpack_scales(p, cols):
    return p.transpose(1, 0, 2).reshape(p.shape[1], -1)[:, : cols // 32]


def ffn_backward_kept(x_rows, z, offsets, w1, w2, act, dy):
    """(dx, dw1, dw2) of the experts' FFN with Z's kept values z [R, d_ff] in the
    place of Z, x_rows the rows that dW1 takes."""
    dx = np.zeros((z.shape[0], w1.shape[2]))
    dw1, dw2 = np.zeros(w1.shape), np.zeros(w2.shape)
    for e in range(w1.shape[0]):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        dz = (dy[r] @ w2[e]) * activation_grad(z[r], act)
        dx[r] = dz @ w1[e]
        dw1[e] = dz.T @ x_rows[r]
        dw2[e] = dy[r].T @ activation(z[r], act)
    return dx, dw1, dw2


# ------------------------------------------------------------ a whole block
def block_forward(p, dec, cfg):
    """o of a block with its decisions held fixed.  p: x, w_gate, b_gate, w1, w2,
    w_pre, b_pre, w_post, b_post, gate (None where there is none); dec: idx,
    slot_pos, rep_row, rep_of_pos, rep_token, rep_offsets; cfg: norm, eps,
    res_scale, score, renormalise, scale, act.  Returns (o, what the backward
    needs)."""
    n = dict(norm=cfg["norm"], eps=cfg["eps"])
    u = pre_norm(p["x"], w_pre=p["w_pre"], b_pre=p["b_pre"], **n)
    l = u @ p["w_gate"].T + p["b_gate"]
    g = gates(l, dec["idx"], cfg["score"], cfg["renormalise"], cfg["scale"])
    off = dec["rep_offsets"]
    R = int(off[-1])
    z = np.zeros((R, p["w1"].shape[1]))
    y_rep = np.zeros((R, u.shape[1]))
    for e in range(len(off) - 1):
        r = slice(int(off[e]), int(off[e + 1]))
        z[r] = u[dec["rep_token"][r]] @ p["w1"][e].T
        y_rep[r] = activation(z[r], cfg["act"]) @ p["w2"][e].T
    kept = dec["slot_pos"] >= 0
    row = np.where(kept, dec["rep_row"][np.maximum(dec["slot_pos"], 0)], 0)
    y = (np.where(kept, g, 0.0)[..., None] * y_rep[row]).sum(1) if R else np.zeros_like(u)
    o = block_norm(p["x"], y, res_scale=cfg["res_scale"], w_post=p["w_post"], b_post=p["b_post"], gate=p["gate"], **n)
    return o, dict(u=u, l=l, g=g, z=z, y_rep=y_rep, y=y, o=o, row=row, kept=kept)


def block_backward(p, dec, cfg, s, dout, dlogits=None):
    """Gradients of block_forward (a dict: dx, dw_gate, ...) from what it left."""
    n = dict(norm=cfg["norm"], eps=cfg["eps"])
    out = block_norm_backward(s["y"], s["o"], dout, None, res_scale=cfg["res_scale"], w_post=p["w_post"],
                              b_post=p["b_post"], gate=p["gate"], **n)
    stream, dy = out.pop("dx"), out.pop("dy")
    dg = np.where(s["kept"], (dy[:, None] * s["y_rep"][s["row"]]).sum(2), 0.0)
    dy_rep = np.zeros_like(s["y_rep"])
    for j in range(dg.shape[1]):
        np.add.at(dy_rep, s["row"][s["kept"][:, j], j], (s["g"][:, j, None] * dy)[s["kept"][:, j]])
    dx_rep, out["dw1"], out["dw2"] = ffn_backward_kept(s["u"][dec["rep_token"]], s["z"], dec["rep_offsets"], p["w1"],
                                                       p["w2"], cfg["act"], dy_rep)
    du, out["dw_gate"], out["db_gate"] = route_backward(
        s["u"], p["w_gate"], s["l"], dec["idx"], dg, cfg["score"], cfg["renormalise"], cfg["scale"], dlogits, dx_rep,
        dec["slot_pos"], dec["rep_of_pos"], dec["rep_row"])
    pre = block_norm_backward(None, p["x"], stream, du, norm=cfg["norm"], eps=cfg["eps"], w_pre=p["w_pre"])
    out.update(dx=pre["dx"], dw_pre=pre["dw_pre"], db_pre=pre["db_pre"])
    return out


__all__ = [n for n in dir() if not n.startswith("_") and n not in ("annotations", "math", "np")]
