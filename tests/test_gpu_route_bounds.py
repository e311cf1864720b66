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


# ------------------------------------------------------- what the instructions round
# The kernels' bound in units of 2^-24 |x| |w|.  Four K steps are one chain of sums: 64
# float32 products, each a rounding, or 128 bf16 ones, of which every eight are, and which
# lose eight units more together, being cut off 2^-24 below the largest of their eight.
# Then a rounding a chain (a wave of the block kernels has a quarter of the columns), and
# 5 or 2 for what joins these sums.
def roundings(dtype, T, d, E):
    chains = lambda steps: (steps + 3) // 4  # noqa: E731
    if dtype == "f32":
        return 64 + chains((d // 16 + 3) // 4) + 5
    if T >= 32768 and E * d * 2 <= 128 * 1024:
        return 16 + 8 + chains(d // 32) + 2
    return 16 + 8 + chains((d // 32 + 3) // 4) + 5


def within(logits, x, w, b, dtype, T):
    """|logit - exact| by the bound for the gate weights of the largest norm, as the
    router applies it, and the last rounding of a logit that was taken again."""
    l = exact(x, w, b)
    norms = np.linalg.norm(x.double().cpu().numpy(), axis=1)[:, None] * np.linalg.norm(w.double().cpu().numpy(), axis=1).max()
    room = 1.01 * roundings(dtype, T, x.shape[1], w.shape[0]) * U * norms + U * np.abs(l)
    if b is not None:
        room = room + 2 * U * float(b.abs().max())
    err = np.abs(logits.double().cpu().numpy() - l)
    assert (err <= room).all(), float((err / room).max())


@pytest.mark.parametrize("dtype,T,d,E", KERNELS + [("bf16", 32768, 512, 24), ("bf16", 40000, 2048, 32), ("f32", 300, 4096, 64),
                                                   ("bf16", 300, 4096, 64), ("f32", 17, 64, 3), ("bf16", 5, 64, 3)])
@pytest.mark.parametrize("rows", ["normal", "positive", "cancelling"])
def test_logits_within_the_bound_that_choices_rest_on(rows, dtype, T, d, E):
    rng = np.random.default_rng(d)
    n = min(T, 256)
    x, w = rng.standard_normal((n, d)), rng.standard_normal((E, d))
    if rows == "positive":
        x, w = np.abs(x), np.abs(w) + 1.0
    if rows == "cancelling":
        x[:, d // 2:], w[:, d // 2:] = -x[:, :d // 2], w[:, :d // 2]
    x, w = tensor(x, dtype), tensor(w, dtype)
    idx, logits = route(x[np.arange(T) % n].contiguous(), w, None, 2)
    within(logits[:n], x, w, None, dtype, T)
    l = exact(x, w, None)
    got, want = idx[:n].cpu().numpy(), best(l, 2)
    if dtype == "bf16":      # (products of 16 bits: float64 sums of theirs are exact)
        assert np.array_equal(got, want)
    else:                    # both sides' float64 sums are within d 2^-53 |x| |w| of the exact ones
        slack = 2 * d * 2.0 ** -53 * np.linalg.norm(x.double().cpu().numpy(), axis=1) * np.linalg.norm(
            w.double().cpu().numpy(), axis=1).max()
        differ = np.abs(np.take_along_axis(l, got, 1) - np.take_along_axis(l, want, 1))
        assert (differ <= 2 * slack[:, None]).all() and (got[:, 0] != got[:, 1]).all()


def check_pair(dtype, T, E, x, a, b, bias):
    """The expert 5 with weights a, chosen before 2 with b, of rows that are all x; the
    others have none."""
    d = len(x)
    w = np.zeros((E, d))
    w[5], w[2] = a, b
    x, w = tensor(x[None], dtype), tensor(w, dtype)
    bias = None if bias is None else bias * tensor(np.ones(E), "f32")
    l = exact(x, w, bias)
    assert l[0, 5] > l[0, 2] > np.delete(l[0], [2, 5]).max()
    idx, logits = route(x.expand(T, d).contiguous(), w, bias, 2)
    within(logits[:3], x, w, bias, dtype, T)
    assert np.array_equal(idx.cpu().numpy(), np.broadcast_to([5, 2], (T, 2)))


@pytest.mark.parametrize("T,E", [(40, 8), (9001, 8), (33001, 8)])
def test_float32_products_that_round_one_by_one(T, E):
    """A sum that stays at 1 under 1023 products of just less than half a unit each: 6.1e-5
    in all, beside a rival at 1 + 5.4e-5."""
    x = np.zeros(4096)
    x[0], x[1:1024] = 1.0, np.float32(0.9975 * 2.0 ** -12)
    rival = np.zeros(4096)
    rival[0] = np.float32(1 + 5.4e-5)
    check_pair("f32", T, E, x, x, rival, None)


@pytest.mark.parametrize("T,E", [(40, 8), (9001, 24), (33001, 24)])
def test_bf16_products_that_round_by_eights(T, E):
    """The same with eight products just below half a unit, which a bias of -1 brings to
    light: 126 units of 2^-24 that the sum does not see, beside a rival of 110."""
    x, a, b = np.zeros(4096), np.zeros(4096), np.zeros(4096)
    x[0], x[1:1024], x[1024] = 1.0, 2.0 ** -13, 2.0 ** -9
    a[0], a[1:1024] = 1.0, 253 / 256 * 2.0 ** -14
    b[0], b[1024] = 1.0, 110 * 2.0 ** -15
    check_pair("bf16", T, E, x, a, b, -1.0)


@pytest.mark.parametrize("T", [32768, 33001])
def test_bf16_products_of_the_streaming_kernel(T):
    """256 columns are one sum there: one expert's loses 31 units, its rival's, just above
    half a unit, wins 30."""
    x, a, b = np.zeros(512), np.zeros(512), np.zeros(512)
    x[0], x[1:256], x[256] = 1.0, 2.0 ** -13, 2.0 ** -9
    a[0], a[1:256] = 1.0, 253 / 256 * 2.0 ** -14
    b[0], b[1:256], b[256] = 1.0, 131 / 128 * 2.0 ** -14, -4 * 2.0 ** -15
    check_pair("bf16", T, 8, x, a, b, -1.0)
