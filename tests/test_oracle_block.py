"""The 64-bit forms of a block's operators: gradients against differences, the
8-bit format against its definition (CPU)."""
import itertools

import numpy as np
import pytest

from oracle import block_oracle as B


def slope(f, a, at, h=1e-6):
    """df/da[at] by a central difference."""
    up, down = a.copy(), a.copy()
    up[at] += h
    down[at] -= h
    return (f(up) - f(down)) / (2 * h)


def check(f, a, grad, rng, places=6):
    """grad is that of f at a: truncation of the difference is O(h^2) = 1e-12,
    its rounding O(1e-16 / h) = 1e-10 of the sums of some hundred terms of
    order one."""
    for _ in range(places):
        at = tuple(rng.integers(0, n) for n in a.shape)
        assert abs(slope(f, a, at) - grad[at]) < 1e-6 * max(1.0, abs(grad[at])), at


@pytest.mark.parametrize("norm,post,gate,pre", itertools.product(("rms", "layer"), (0, 1), (0, 1, 2), (0, 1)))
def test_block_norm_gradients(norm, post, gate, pre):
    rng = np.random.default_rng(3)
    T, d = 5, 24
    p = dict(x=rng.standard_normal((T, d)), y=rng.standard_normal((T, d)) + 0.3)
    if post:
        p.update(w_post=rng.standard_normal(d), b_post=rng.standard_normal(d))
    if gate:
        p["gate"] = rng.standard_normal(d) if gate == 1 else rng.standard_normal((T, d))
    if pre:
        p.update(w_pre=rng.standard_normal(d), b_pre=rng.standard_normal(d))
    do, du = rng.standard_normal((T, d)), rng.standard_normal((T, d))
    kw = dict(norm=norm, eps=1e-3)

    def loss(p):
        o = B.block_norm(p["x"], p["y"], res_scale=0.7, w_post=p.get("w_post"), b_post=p.get("b_post"),
                         gate=p.get("gate"), **kw)
        f = (do * o).sum()
        return f + (du * B.pre_norm(o, w_pre=p["w_pre"], b_pre=p["b_pre"], **kw)).sum() if pre else f

    o = B.block_norm(p["x"], p["y"], res_scale=0.7, w_post=p.get("w_post"), b_post=p.get("b_post"), gate=p.get("gate"),
                     **kw)
    g = B.block_norm_backward(p["y"], o, do, du if pre else None, res_scale=0.7, w_post=p.get("w_post"),
                              b_post=p.get("b_post"), gate=p.get("gate"), w_pre=p.get("w_pre"), **kw)
    for name in p:
        check(lambda a: loss(dict(p, **{name: a})), p[name], g["d" + name], rng)


@pytest.mark.parametrize("score,renorm,k", itertools.product(("softmax", "sigmoid"), (False, True), (1, 3)))
def test_route_gradients(score, renorm, k):
    rng = np.random.default_rng(5)
    T, E, d = 6, 8, 12
    x, w, b = rng.standard_normal((T, d)), 0.3 * rng.standard_normal((E, d)), rng.standard_normal(E)
    idx = B.choose(x @ w.T + b, k, score)
    dgate, extra = rng.standard_normal((T, k)), 0.1 * rng.standard_normal((T, E))

    def loss(x, w, b):
        l = x @ w.T + b
        return (dgate * B.gates(l, idx, score, renorm, 1.5)).sum() + (extra * l).sum()

    dx, dw, db = B.route_backward(x, w, x @ w.T + b, idx, dgate, score, renorm, 1.5, extra)
    check(lambda a: loss(a, w, b), x, dx, rng)
    check(lambda a: loss(x, a, b), w, dw, rng)
    check(lambda a: loss(x, w, a), b, db, rng)


def test_choice_by_groups():
    l = np.array([[1.0, 0.9, 3.0, -5.0, 2.0, 1.9, 0.0, 0.0]])
    # one best a group: groups of 2 hold 1.0, 3.0, 2.0, 0.0
    assert B.choose(l, 2, "sigmoid", groups=4, top_groups=2, group_best=1).tolist() == [[2, 4]]
    # two best (of the scores): the pair of 2.0 and 1.9 before that of 1.0 and 0.9, 3.0 and -5.0 last but one
    assert B.choose(l, 2, "sigmoid", groups=4, top_groups=2, group_best=2).tolist() == [[4, 5]]
    # ties: the lower index; a bias reverses the choice but is no part of the gate
    assert B.choose(np.zeros((1, 4)), 2, "softmax").tolist() == [[0, 1]]
    idx = B.choose(np.zeros((1, 4)), 2, "softmax", balance=np.array([0.0, 0.1, 0.0, 0.2]))
    assert idx.tolist() == [[3, 1]] and np.allclose(B.gates(np.zeros((1, 4)), idx, "softmax", False), 0.25)


def test_mx8_format():
    rng = np.random.default_rng(7)
    x = rng.standard_normal((50, 96)) * np.exp(3 * rng.standard_normal((50, 3))).repeat(32, 1)
    q, s = B.mx8_quantize(x)
    v = B.mx8_values(q, s)
    step = np.ldexp(1.0, s.astype(int) - 127).repeat(32, 1)
    most = np.abs(x.reshape(50, 3, 32)).max(-1).repeat(32, 1)
    assert (most < 128 * step).all() and (most >= 64 * step).all()
    # half a step, but for values between 127 and 128 steps, which become 127
    assert (np.abs(v - x) <= np.where(np.abs(x) > 127.5 * step, 1.0, 0.5) * step).all()
    assert np.array_equal(B.mx8_rounded(v), v)
    assert np.array_equal(v, v.astype(np.float32)) and (np.abs(q) <= 127).all()
    odd = np.zeros((1, 96))
    odd[0, 3], odd[0, 40], odd[0, 64:] = 2.0 ** -149, np.inf, np.float64(np.finfo(np.float32).max)
    q, s = B.mx8_quantize(odd)
    assert s.tolist() == [[0, 255, 248]] and q[0, 3] == 0 and (q[0, 64:] == 127).all()
    assert np.isnan(B.mx8_values(q, s)[0, 32:64]).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_kept_ffn_gradients(act):
    rng = np.random.default_rng(9)
    E, d, f = 2, 6, 8
    off = np.array([0, 3, 5])
    x, w1, w2 = rng.standard_normal((5, d)), rng.standard_normal((E, f, d)), rng.standard_normal((E, d, f))
    dy = rng.standard_normal((5, d))
    e_of = np.repeat(np.arange(E), np.diff(off))

    def loss(x, w1, w2):
        return sum((dy[r] * (w2[e] @ B.activation(w1[e] @ x[r], act))).sum() for r, e in enumerate(e_of))

    z = np.stack([w1[e] @ x[r] for r, e in enumerate(e_of)])
    dx, dw1, dw2 = B.ffn_backward_kept(x, z, off, w1, w2, act, dy)
    check(lambda a: loss(a, w1, w2), x, dx, rng)
    check(lambda a: loss(x, a, w2), w1, dw1, rng)
    check(lambda a: loss(x, w1, a), w2, dw2, rng)


@pytest.mark.parametrize("norm,score,renorm", [("rms", "sigmoid", True), ("layer", "softmax", False)])
def test_block_gradients(norm, score, renorm):
    rng = np.random.default_rng(11)
    T, d, E, k, f = 6, 8, 4, 3, 10
    p = dict(x=rng.standard_normal((T, d)), w_gate=0.3 * rng.standard_normal((E, d)), b_gate=rng.standard_normal(E),
             w1=rng.standard_normal((E, f, d)), w2=rng.standard_normal((E, d, f)), w_pre=1 + 0.1 * rng.standard_normal(d),
             b_pre=0.1 * rng.standard_normal(d), w_post=1 + 0.1 * rng.standard_normal(d),
             b_post=0.1 * rng.standard_normal(d), gate=rng.standard_normal(d))
    cfg = dict(norm=norm, eps=1e-3, res_scale=0.8, score=score, renormalise=renorm, scale=1.5, act="gelu")
    u = B.pre_norm(p["x"], norm=norm, eps=1e-3, w_pre=p["w_pre"], b_pre=p["b_pre"])
    idx = B.choose(u @ p["w_gate"].T + p["b_gate"], k, score)
    slot_pos, perm, off = B.buckets(idx, E, 0.9)
    rep = rng.random(len(perm)) < 0.6
    rep[off[:-1][off[:-1] < len(perm)]] = True
    rep_of = np.maximum.accumulate(np.where(rep, np.arange(len(perm)), -1))
    dec = dict(idx=idx, slot_pos=slot_pos, rep_of_pos=rep_of, rep_row=(np.cumsum(rep) - 1)[rep_of],
               rep_token=perm[rep], rep_offsets=np.concatenate([[0], np.cumsum(rep)])[off])
    dout, dl = rng.standard_normal((T, d)), 0.1 * rng.standard_normal((T, E))

    def loss(p):
        o, s = B.block_forward(p, dec, cfg)
        return (dout * o).sum() + (dl * s["l"]).sum()

    g = B.block_backward(p, dec, cfg, B.block_forward(p, dec, cfg)[1], dout, dl)
    for name in p:
        check(lambda a: loss(dict(p, **{name: a})), p[name], g["d" + name], rng)
