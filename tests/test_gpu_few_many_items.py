"""luffy_moe_few where a block of the products has several work items one after
the other, of experts with one to 64 columns, whose columns come in several
chunks of K: against the 64-bit layer."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24     # half a unit in the last place of float32, relative


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def act64(z, act):
    import torch
    return z * torch.special.ndtr(z) if act == "gelu" else z * torch.sigmoid(z)


def run_and_compare(w, loads, d, d_ff, act, seed):
    """Every token's first expert is 0; the second ones are spread by `loads`
    (columns of experts 1, 2, ...; None: k = 1)."""
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.float32 if w == "f32" else torch.bfloat16
    T = 64
    E = 1 + len(loads)
    second = np.repeat(np.arange(1, E), loads)
    assert len(second) == T
    second = np.random.default_rng(seed).permutation(second)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    x = normal(T, d)
    x[:, :E] = 0.0
    x[:, 0] = 8.0
    x[torch.arange(T), torch.from_numpy(second)] = 7.0
    x = x.to(t)
    w_gate = torch.eye(E, d, device="cuda").to(t)
    w1, w2 = (0.05 * normal(E, d_ff, d)).to(t), (0.05 * normal(E, d, d_ff)).to(t)
    scales = [None, None]
    v1, v2 = w1, w2
    if w == "mx4":
        (w1, s1), (w2, s2) = L.mx4_weights(w1), L.mx4_weights(w2)
        scales = [s1, s2]
        v1, v2 = torch.empty_like(v1, dtype=torch.float32), torch.empty_like(v2, dtype=torch.float32)
        L.luffy_mx4_dequantize(w1, s1, v1)
        L.luffy_mx4_dequantize(w2, s2, v2)
    idx, gate = torch.empty(T, 2, dtype=torch.int32, device="cuda"), torch.empty(T, 2, device="cuda")
    y = torch.full((T, d), 768.0, dtype=t, device="cuda")
    ws = torch.full((L.moe_few_workspace_size(T, d, E, 2, d_ff),), 0xFF, dtype=torch.uint8, device="cuda")
    L.luffy_moe_few(x, w_gate, None, w1, w2, 2, act, idx, gate, y, ws, w1_scale=scales[0], w2_scale=scales[1])
    assert (idx[:, 0] == 0).all() and np.array_equal(idx[:, 1].cpu().numpy(), second)
    g = torch.softmax(torch.tensor([8.0, 7.0], dtype=torch.float64), 0).tolist()
    assert (gate.double() - torch.tensor(g, dtype=torch.float64, device="cuda")).abs().max().item() <= 8 * U32
    ref, bound = torch.zeros(T, d, dtype=torch.float64, device="cuda"), torch.zeros(T, d, dtype=torch.float64, device="cuda")
    for j in (0, 1):
        for e in range(E):
            rows = torch.from_numpy(np.flatnonzero((second if j else 0 * second) == e)).cuda()
            if rows.numel() == 0:
                continue
            xe, a, b = x[rows].double(), v1[e].double(), v2[e].double()
            h = act64(xe @ a.t(), act)
            # first product: d float32 additions, |act'| <= 1.13; what a hidden value is
            # kept as; second product: d_ff additions (of up to three parts); the gate
            eh = 1.13 * d * U32 * (xe.abs() @ a.abs().t()) + 16 * U32 * h.abs()
            if w == "bf16":
                eh += 2.0 ** -17 * h.abs()
            if w == "mx4":
                top = h.abs().reshape(h.shape[0], -1, 32).amax(-1).repeat_interleave(32, dim=1)
                eh += 2.0 ** -12 * h.abs() + 2.0 ** -25 * top
            ref[rows] += g[j] * (h @ b.t())
            bound[rows] += g[j] * (eh @ b.abs().t() + (3 * d_ff + 32) * U32 * (h.abs() @ b.abs().t()))
    got = y.double()
    low, high = (ref - bound).to(t).double(), (ref + bound).to(t).double()
    bad = ~((got >= low) & (got <= high))
    assert not bad.any().item(), (bad.nonzero()[:4].tolist(), (got - ref).abs().max().item())
    # and all together far closer than the sum of all worst cases: the result's own
    # rounding, at most 2^-8 of it in bf16, and sums whose errors mostly cancel
    assert ((got - ref).norm() / ref.norm()).item() <= (1e-5 if w == "f32" else 2.0 ** -8)


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("loads", [
    [33, 17, 9, 3, 1, 1, 0],           # eight, four, two and one group of columns, an idle expert
    [16, 16, 10, 9, 8, 5, 0]])
def test_first_product(loads, w):
    """9600 hidden rows: 75 items an expert, 525 in all for 256 blocks."""
    run_and_compare(w, loads, 1088, 9600, "gelu", seed=1)


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("loads", [[33, 17, 9, 3, 1, 1, 0], [32, 18, 14]])
def test_second_product(loads, w):
    run_and_compare(w, loads, 9600, 1088, "silu", seed=2)


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
def test_parts_of_k_and_two_items(w):
    """3200 rows: 25 items an expert would leave CUs idle, so K goes to two waves
    (17 pieces to eight and nine), 350 items for 256 blocks."""
    run_and_compare(w, [33, 17, 9, 3, 1, 1, 0], 1088, 3200, "gelu", seed=3)
    run_and_compare(w, [33, 17, 9, 3, 1, 1, 0], 3200, 1088, "silu", seed=4)


@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 9])
def test_the_last_expert_past_4_gib(w, T):
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(T)
    E, d, d_ff = (64, 4096, 11008) if w == "bf16" else (9, 32768, 32768)
    x = torch.randn(T, d, generator=gen, device="cuda").to(torch.bfloat16)
    w_gate = torch.zeros(E, d, dtype=torch.bfloat16, device="cuda")
    b_gate = torch.full((E,), -50.0, device="cuda")
    b_gate[E - 1] = 50.0
    scales = [None, None]
    if w == "bf16":
        w1, w2 = (torch.zeros(E, *m, dtype=torch.bfloat16, device="cuda") for m in ((d_ff, d), (d, d_ff)))
        for m in (w1, w2):
            m[E - 1].normal_(0, 0.02, generator=gen)
        v1, v2 = w1[E - 1].double(), w2[E - 1].double()
    else:
        w1, w2 = (torch.zeros(E, a, b // 2, dtype=torch.uint8, device="cuda") for a, b in ((d_ff, d), (d, d_ff)))
        scales = [torch.full((E, b // 256, a, 8), 120, dtype=torch.uint8, device="cuda") for a, b in ((d_ff, d), (d, d_ff))]
        v = []
        for q, s in zip((w1, w2), scales):
            q[E - 1] = torch.randint(0, 256, q[0].shape, dtype=torch.uint8, device="cuda", generator=gen)
            s[E - 1] = torch.randint(112, 120, s[0].shape, dtype=torch.uint8, device="cuda", generator=gen)
            f = torch.empty(q.shape[1], 2 * q.shape[2], device="cuda")
            L.luffy_mx4_dequantize(q[E - 1], s[E - 1], f)
            v.append(f.double())
        v1, v2 = v
    idx, gate = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
    y = torch.empty_like(x)
    ws = torch.empty(L.moe_few_workspace_size(T, d, E, 1, d_ff), dtype=torch.uint8, device="cuda")
    L.luffy_moe_few(x, w_gate, b_gate, w1, w2, 1, "gelu", idx, gate, y, ws, w1_scale=scales[0], w2_scale=scales[1])
    assert (idx == E - 1).all()
    ref = act64(x.double() @ v1.t(), "gelu") @ v2.t()
    assert ((y.double() - ref).norm() / ref.norm()).item() <= 2.0 ** -8


@pytest.mark.parametrize("w", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [3, 8, 30])
def test_hidden_values_keep_their_low_parts(T, w):
    """Each result the difference of two hidden values that nearly agree, so that
    it shows what they are kept as: without the second bf16 part or the third
    E4M3 part it would be off by more than the bound."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(T)
    d, d_ff = 256, 512
    bf16 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)
    x = np.zeros((T, d))
    x[:, 0] = rng.uniform(0.5, 4.0, T)
    x[:, 1:32] = rng.uniform(0.25, 1.0, (T, 31)) * 2.0 ** (-6 if w == "mx4" else -9)
    x = bf16(x)
    w1, w2 = np.zeros((d_ff, d)), np.zeros((d, d_ff))
    n = np.arange(d)
    w1[:, 0] = 1.0
    w1[2 * n + 1, 1 + n % 31] = 1.0
    w2[n, 2 * n], w2[n, 2 * n + 1] = -1.0, 1.0
    g1, g2 = bf16(w1)[None].cuda(), bf16(w2)[None].cuda()
    scales = [None, None]
    if w == "mx4":
        (g1, s1), (g2, s2) = L.mx4_weights(g1), L.mx4_weights(g2)      # exact: zeros and ones
        scales = [s1, s2]
    idx, gate = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
    y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(L.moe_few_workspace_size(T, d, 1, 1, d_ff), dtype=torch.uint8, device="cuda")
    L.luffy_moe_few(x.cuda(), torch.zeros(1, d, dtype=torch.bfloat16, device="cuda"), None, g1, g2, 1, "silu", idx,
                    gate, y, ws, w1_scale=scales[0], w2_scale=scales[1])
    z = x.double().numpy() @ w1.T
    h = z / (1.0 + np.exp(-z))
    ref = h @ w2.T
    both = h @ np.abs(w2).T
    bound = both * ((2.0 ** -17 if w == "bf16" else 2.0 ** -12) + 16 * U32)
    if w == "mx4":
        bound = bound + 2.0 ** -24 * h.max()
    got = y.double().cpu().numpy()
    low, high = (torch.from_numpy(v).to(torch.bfloat16).double().numpy() for v in (ref - bound, ref + bound))
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ref).max(), bound.max())
