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
