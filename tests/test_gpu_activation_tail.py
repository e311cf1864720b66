"""Hidden values far in the activation's negative tail: where a block or a row
holds nothing else, they keep their own relative accuracy."""
import math

import numpy as np
import pytest

from oracle import mx4_oracle as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def gpu(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def act64(z, act):
    """The activation in 64 bits, by the complementary error function, so that
    nothing cancels in the tail."""
    if act == "gelu":
        return 0.5 * z * np.vectorize(math.erfc, otypes=[float])(-z * math.sqrt(0.5))
    return z / (1.0 + np.exp(-z))


def tail_layer(rows, d):
    """x [rows, d] of up to three ones a row and w1 [d, d] whose rows hold one negative
    E2M1 value each, so that every pre-activation is an exact small sum: rows
    of w1 in blocks of 32 with values from -0.5 to -6, products -1.5 to -18."""
    rng = np.random.default_rng(17)
    x = np.zeros((rows, d))
    for r in range(rows):
        x[r, rng.choice(32, 3, replace=False) + 32 * (r % (d // 32))] = 1.0
    w1 = np.empty((d, d))
    for b in range(d // 32):
        low, high = sorted(rng.choice(7, 2)) if b % 3 else (3 + b % 4, 3 + b % 4)
        w1[32 * b:32 * b + 32] = -M.MAGNITUDES[1:][rng.integers(low, high + 1, (32, d))]
    # each row of w1 keeps one block size: the value 6 once a block makes the scale 1
    w1[:, ::32] = -6.0
    x[:, ::32] = 0.0
    return x, w1


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_blocks_of_tail_values_get_their_codes(act):
    """W2 the identity: the results are the rounded hidden values themselves."""
    import torch
    import paper_2411_15419_amd as L
    rows, d = 70, 320
    x, w1 = tail_layer(rows, d)
    z = x @ w1.T
    assert z.max() <= -1.0 and z.min() <= -12.0
    keep = z >= -12.5 if act == "gelu" else z >= -80.0
    h = act64(z, act)
    # GELU: 10^-6 (1 + z^2) and the hardware's exp2 and reciprocal; SiLU: the
    # argument of exp2 rounded twice
    tol = 2e-6 * (1.0 + z * z) if act == "gelu" else 2.0 ** -22 * (2.0 + np.abs(z))
    (q1, s1), (q2, s2) = M.pack(*M.quantize(w1)), M.pack(*M.quantize(np.eye(d)))
    assert np.array_equal(M.rounded(w1), w1)
    y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(L.mx4_expert_ffn_workspace_size(rows, 1, d, d), dtype=torch.uint8, device="cuda")
    L.luffy_mx4_expert_ffn(gpu(x, torch.bfloat16), None, gpu(np.array([0, rows], np.int32)), gpu(q1[None]),
                           gpu(s1[None]), gpu(q2[None]), gpu(s2[None]), act, rows, y, ws)
    got = y.double().cpu().numpy()
    low, high = M.rounded(h * (1 - tol)), M.rounded(h * (1 + tol))
    # blocks whose values are all in the range that is stated
    whole = keep.reshape(rows, -1, 32).all(-1).repeat(32, axis=1)
    assert whole.mean() > 0.5
    bad = whole & ~((got >= np.minimum(low, high)) & (got <= np.maximum(low, high)))
    assert not bad.any(), (np.argwhere(bad)[:4], z[bad][:4], got[bad][:4], h[bad][:4])
    assert (got[whole & (h != 0)] != 0).mean() > 0.5


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("T", [7, 40])
def test_a_step_keeps_tail_values(T, act, w):
    """luffy_moe_few with one expert and W2 the identity: the results are the
    hidden values as the second product holds them."""
    import torch
    import paper_2411_15419_amd as L
    d = 320
    x, w1 = tail_layer(T, d)
    z = x @ w1.T
    h = act64(z, act)
    t = torch.float32 if w == "f32" else torch.bfloat16
    w2 = np.eye(d)
    scales = [None, None]
    if w == "mx4":
        (g1, s1), (g2, s2) = M.pack(*M.quantize(w1)), M.pack(*M.quantize(w2))
        g1, g2, scales = gpu(g1[None]), gpu(g2[None]), [gpu(s1[None]), gpu(s2[None])]
    else:
        g1, g2 = gpu(w1[None], t), gpu(w2[None], t)
    idx, gate = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
    y = torch.empty(T, d, dtype=t, device="cuda")
    ws = torch.empty(L.moe_few_workspace_size(T, d, 1, 1, d), dtype=torch.uint8, device="cuda")
    L.luffy_moe_few(gpu(x, t), torch.zeros(1, d, dtype=t, device="cuda"), None, g1, g2, 1, act, idx, gate, y, ws,
                    w1_scale=scales[0], w2_scale=scales[1])
    got = y.double().cpu().numpy()
    # erfcf's and expf's argument rounded, a few units in the last place; then
    # what the hidden values are kept as, for 4 bits also 2^-25 of their block's
    # largest; then the result's own rounding
    tol = (2.0 * z * z + 16.0) * 2.0 ** -24 + {"f32": 0.0, "bf16": 2.0 ** -17, "mx4": 2.0 ** -12}[w]
    slack = 2.0 ** -126 * np.ones_like(h)
    if w == "mx4":
        slack += 2.0 ** -25 * np.abs(h).reshape(T, -1, 32).max(-1).repeat(32, axis=1)
    low, high = h - tol * np.abs(h) - slack, h + tol * np.abs(h) + slack
    low, high = (torch.from_numpy(v).to(t).double().numpy() for v in (low, high))
    bad = (z >= -12.5) & ~((got >= low) & (got <= high))
    assert not bad.any(), (np.argwhere(bad)[:4], z[bad][:4], got[bad][:4], h[bad][:4])
