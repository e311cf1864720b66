"""Infinities on their way through luffy_moe_few: what the formula makes of them,
whatever the number of tokens."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


@pytest.mark.parametrize("w", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 8, 9, 20, 64])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_overflow_gives_signed_infinities(T, act, w):
    """Token 0's hidden value 437 overflows: its results are infinite with the
    signs of W2's column, the other tokens' are finite."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(T)
    d, d_ff = 320, 448
    t = torch.float32 if w == "f32" else torch.bfloat16
    x = rng.uniform(0.5, 1.0, (T, d))
    w1, w2 = rng.uniform(0.1, 0.2, (d_ff, d)), rng.uniform(0.1, 0.2, (d, d_ff))
    sign = rng.choice([-1.0, 1.0], d)
    x[:, 311] = 0.0
    x[0, 311] = w1[437, 311] = 1e20
    w2[:, 437] *= sign
    gpu = lambda a: torch.from_numpy(a).to(t).cuda()
    idx, gate = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
    y = torch.empty(T, d, dtype=t, device="cuda")
    ws = torch.empty(L.moe_few_workspace_size(T, d, 1, 1, d_ff), dtype=torch.uint8, device="cuda")
    w_gate = torch.zeros(1, d, dtype=t, device="cuda")
    L.luffy_moe_few(gpu(x), w_gate, None, gpu(w1[None]), gpu(w2[None]), 1, act, idx, gate, y, ws)
    got = y.double().cpu().numpy()
    assert np.array_equal(got[0], np.inf * sign)
    assert np.isfinite(got[1:]).all()
