"""Plain 64-bit forms of the serving operators: microscaled 4-bit matrices,
their product, the experts' FFN on them and a layer's step of a few tokens.
Written from the definitions in include/luffy.h; numpy only."""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_e2m1(u):
    """Codes (0..15) of the nearest representable values, halfway cases to the
    even code, by distance to each of the eight magnitudes."""
    a = np.abs(np.asarray(u, np.float64))
    dist = np.abs(a[..., None] - MAGNITUDES)
    near = dist.min(-1, keepdims=True)
    odd_last = np.where(dist == near, np.arange(8) % 2, 2)     # even codes first among equals
    code = odd_last.argmin(-1)
    return (code + 8 * np.signbit(u)).astype(np.uint8)


def quantize(x):
    """x [rows, cols] -> codes [rows, cols], scale bytes [rows, cols/32]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    b = x.reshape(rows, cols // 32, 32)
    finite = np.isfinite(b).all(-1)
    most = np.abs(np.where(finite[..., None], b, 0.0)).max(-1)
    e = np.full(most.shape, -127, np.int64)
    nz = most > 0
    e[nz] = np.maximum(np.frexp(most[nz])[1] - 1 - 2, -127)
    code = round_e2m1(np.where(finite[..., None], b, 0.0) / np.ldexp(1.0, e)[..., None])
    code[~finite] = 0
    s = np.where(finite, e + 127, 255).astype(np.uint8)
    s[finite & ~nz] = 0
    return code.reshape(rows, cols), s


def values(code, s):
    """The values of codes [rows, cols] under scale bytes [rows, cols/32]."""
    v = np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    f = np.ldexp(1.0, s.astype(np.int64) - 127)
    f = np.where(s == 255, np.nan, f)
    return v * np.repeat(f, 32, axis=-1)


def rounded(x):
    return values(*quantize(x))


def pack(code, s):
    """The stored form: values [rows, cols/2], scales [ceil(cols/256), rows, 8]."""
    rows, n = s.shape
    q = code[:, 0::2] | (code[:, 1::2] << 4)
    p = np.zeros((rows, (n + 7) // 8 * 8), np.uint8)
    p[:, :n] = s
    return q, np.ascontiguousarray(p.reshape(rows, -1, 8).transpose(1, 0, 2))


def activation(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + np.vectorize(math.erf, otypes=[float])(z * math.sqrt(0.5)))
    return z / (1.0 + np.exp(-np.maximum(z, -700.0)))


def gate(x, w_gate, b_gate, k):
    """(experts [T, k], gates [T, k], logits): descending logits, ties to the
    lower index; softmax probability (k = 1) or the two renormalised."""
    logits = x @ w_gate.T + (0.0 if b_gate is None else b_gate)
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(logits, idx, 1)
    if k == 1:
        g = 1.0 / np.exp(logits - top).sum(1, keepdims=True)
    else:
        g = np.exp(top - top.max(1, keepdims=True))
        g = g / g.sum(1, keepdims=True)
    return idx, g, logits


def moe(x, w_gate, b_gate, w1, w2, k, act):
    """The layer without condensation: outputs, experts, gates, and for every
    output the sum of the absolute values of its terms, of their second factors'
    errors' weights (for error bounds)."""
    idx, g, _ = gate(x, w_gate, b_gate, k)
    T, d = x.shape
    y = np.zeros((T, d))
    terms = np.zeros((T, d))       # sum |g w2 h|
    spread = np.zeros((T, d))      # sum |g w2| sum |w1 x|
    for t in range(T):
        for j in range(k):
            e = idx[t, j]
            z = w1[e] @ x[t]
            h = activation(z, act)
            y[t] += g[t, j] * (w2[e] @ h)
            terms[t] += g[t, j] * (np.abs(w2[e]) @ np.abs(h))
            spread[t] += g[t, j] * (np.abs(w2[e]) @ (np.abs(w1[e]) @ np.abs(x[t])))
    return y, idx, g, terms, spread
