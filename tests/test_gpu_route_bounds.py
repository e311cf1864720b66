"""Rows at which a float32 sum says little about the logit: whether the scored router
knows it, in every kernel that makes logits, and decides them from exact products."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a unit in the last place of float32, relative
# dtype, T, d, E of every kernel that makes logits: one launch with the choices, blocks
# of 32 and of 64 tokens, and the streaming one (bf16 weights that fit LDS, 128 tokens a
# CU and more)
KERNELS = [("bf16", 40, 512, 8), ("bf16", 9001, 512, 8), ("bf16", 33001, 2112, 40), ("bf16", 33001, 512, 8),
           ("f32", 40, 512, 8), ("f32", 9001, 512, 8), ("f32", 33001, 512, 8)]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def route(x, w, b, k, score="softmax"):
    """(choices, logits) of x [T, d], w [E, d], b [E] or None."""
    import torch
    import paper_2411_15419_amd as L
    (T, _), E = x.shape, w.shape[0]
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    idx, logits = torch.full((T, k), -7, **i32), torch.full((T, E), -7.0, **f32)
    ws = torch.empty(L.route_workspace_size(T, E, k), dtype=torch.uint8, device="cuda")
    L.luffy_route_scored(x, w, b, k, score, 0.0, idx, torch.empty(T, k, **f32), logits, torch.empty(T, k, **i32),
                         torch.empty(T * k, **i32), torch.empty(E + 1, **i32), ws)
    return idx, logits


def exact(x, w, b):
    """Logits of a few rows in float64, which holds these sums to 2^-53 of |x| |w|."""
    l = x.double().cpu().numpy() @ w.double().cpu().numpy().T
    return l if b is None else l + b.double().cpu().numpy()


def best(l, k):
    """The k largest, the lower index first among equal ones."""
    return np.argsort(-l, axis=1, kind="stable")[:, :k]


def tensor(a, dtype):
    import torch
    return torch.from_numpy(a).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()


@pytest.mark.parametrize("dtype,T,d,E", KERNELS)
@pytest.mark.parametrize("of_x,of_w", [(0, 0), (-80, 0), (0, -80), (-100, 20), (-45, -45), (-64, -64), (-110, 0)])
def test_tiny_rows_that_cancel(of_x, of_w, dtype, T, d, E):
    """A sum whose last term is lost beside two large ones that cancel: the same choice
    whatever power of two the rows or the weights are scaled by, also where the squares
    of their values are below float32's smallest."""
    x, w = np.zeros((3, d)), np.zeros((E, d))
    x[:, 0], x[:, 128], x[:, 256], x[:, 300] = 64, 1, 64, 1
    x[1] *= -1                                             # the other order
    x[2, 128] = 0                                          # nothing is lost
    w[:, 300] = -np.arange(1, E + 1) / 16.0                # below the two that compete, in order
    w[2, 0], w[2, 256], w[2, 128], w[2, 300] = 16, -16, 2.0 ** -15, 0     # 2^-15, but 0 in float32
    w[5, 300] = 2.0 ** -16
    x, w = tensor(np.ldexp(x, of_x), dtype), tensor(np.ldexp(w, of_w), dtype)
    want = best(exact(x, w, None), 3)
    assert want[0].tolist() == [2, 5, 0] and want[2].tolist() == [5, 2, 0]
    rows = np.random.default_rng(1).integers(0, 3, T)
    idx, _ = route(x[rows].contiguous(), w, None, 3)
    assert np.array_equal(idx.cpu().numpy(), want[rows])


def test_zero_rows_with_a_bias():
    """Rows of zeros (padding) go by the bias alone, zero weights too."""
    import torch
    for T in (5, 700, 9001, 33001):
        x, w = torch.zeros(T, 256, dtype=torch.bfloat16, device="cuda"), torch.zeros(16, 256, dtype=torch.bfloat16,
                                                                                     device="cuda")
        b = torch.randperm(16, generator=torch.Generator().manual_seed(T)).float().cuda() / 16
        for t in (w, w + 1):
            idx, logits = route(x, t, b, 4)
            assert bool((idx == torch.argsort(b, descending=True)[:4]).all()) and bool((logits == b).all())
