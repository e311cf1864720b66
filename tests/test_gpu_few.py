"""A layer's step of a few tokens (luffy_moe_few) against its 64-bit form."""
import numpy as np
import pytest

from oracle import mx4_oracle as M

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24     # half a unit in the last place of float32, relative


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


def as_type(a, w):
    """Values of a as the activations' type holds them, in 64 bits."""
    import torch
    t = torch.from_numpy(np.asarray(a, np.float32))
    return (t if w == "f32" else t.to(torch.bfloat16)).double().numpy()


class Layer:
    """Weights of a layer on both sides."""

    def __init__(self, rng, w, E, d, d_ff, bias=True):
        import torch
        self.w, self.E, self.d, self.d_ff = w, E, d, d_ff
        self.t = torch.float32 if w == "f32" else torch.bfloat16
        self.w_gate = as_type(0.1 * rng.standard_normal((E, d)), w)
        self.b_gate = rng.standard_normal(E).astype(np.float32) * 0.1 if bias else None
        w1, w2 = 0.05 * rng.standard_normal((E, d_ff, d)), 0.05 * rng.standard_normal((E, d, d_ff))
        self.s1 = self.s2 = None
        if w == "mx4":
            m1, m2 = [M.quantize(m) for m in w1], [M.quantize(m) for m in w2]
            self.w1, self.w2 = np.stack([M.values(*m) for m in m1]), np.stack([M.values(*m) for m in m2])
            (q1, s1), (q2, s2) = (map(np.stack, zip(*[M.pack(*m) for m in ms])) for ms in (m1, m2))
            self.g1, self.g2, self.s1, self.s2 = gpu(q1), gpu(q2), gpu(s1), gpu(s2)
        else:
            self.w1, self.w2 = as_type(w1, w), as_type(w2, w)
            self.g1, self.g2 = gpu(self.w1, self.t), gpu(self.w2, self.t)
        self.gg = gpu(self.w_gate, self.t)
        self.gb = None if self.b_gate is None else gpu(self.b_gate)

    def buffers(self, T, k):
        import torch
        import paper_2411_15419_amd as L
        return dict(idx=torch.full((T, k), -7, dtype=torch.int32, device="cuda"),
                    gate=torch.full((T, k), -7.0, device="cuda"),
                    y=torch.full((T, self.d), 768.0, dtype=self.t, device="cuda"),
                    ws=torch.full((L.moe_few_workspace_size(T, self.d, self.E, k, self.d_ff),), 0xFF,
                                  dtype=torch.uint8, device="cuda"))

    def call(self, x, k, act, b, stream=None):
        import paper_2411_15419_amd as L
        L.luffy_moe_few(x, self.gg, self.gb, self.g1, self.g2, k, act, b["idx"], b["gate"], b["y"], b["ws"],
                        w1_scale=self.s1, w2_scale=self.s2, stream=stream)

    def check(self, x, k, act, b, rows=None):
        """Compares the buffers with the 64-bit layer on x (rows: only these)."""
        y, idx, g, terms, spread = M.moe(x, self.w_gate, self.b_gate, self.w1, self.w2, k, act)
        rows = np.arange(x.shape[0]) if rows is None else np.asarray(rows)
        assert np.array_equal(b["idx"].cpu().numpy()[rows], idx[rows])
        gate = b["gate"].double().cpu().numpy()
        # a few float32 operations (expf, divisions, a sum of at most 64 terms)
        assert np.abs(gate - g)[rows].max() <= 80 * U32
        # first product: d float32 additions, |act'| <= 1.13; hidden value: a few
        # ulp, and its two bf16 parts 2^-17; second product: d_ff additions (two
        # products a value); gates
        bound = 1.13 * self.d * U32 * spread + (2 * self.d_ff + 100) * U32 * terms + 8 * U32 * spread
        if self.w != "f32":
            bound = bound + 2.0 ** -17 * terms
        # the result is what a value within the bound rounds to in its type
        import torch
        got = b["y"].double().cpu().numpy()
        low, high = (torch.from_numpy(v).to(self.t).double().numpy() for v in (y - bound, y + bound))
        bad = ~((got >= low) & (got <= high))[rows]
        assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - y)[rows].max())


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("T,E,k,d,d_ff,act", [
    (1, 1, 1, 64, 64, "gelu"), (1, 4, 2, 256, 320, "silu"), (2, 3, 1, 192, 128, "gelu"), (7, 13, 2, 128, 576, "silu"),
    (8, 4, 1, 320, 256, "gelu"), (9, 2, 2, 64, 192, "gelu"), (17, 5, 2, 576, 64, "silu"), (33, 64, 2, 128, 128, "gelu"),
    (64, 2, 2, 192, 320, "silu"), (64, 64, 1, 64, 256, "gelu"), (25, 3, 1, 512, 1088, "gelu"),
    (5, 8, 2, 1024, 512, "silu")])
def test_layer(T, E, k, d, d_ff, act, w):
    import torch
    rng = np.random.default_rng(T * 1009 + E * 31 + d + d_ff)
    layer = Layer(rng, w, E, d, d_ff, bias=T % 2 == 1)
    x = as_type(rng.standard_normal((T, d)), w)
    b = layer.buffers(T, k)
    layer.call(gpu(x, layer.t), k, act, b)
    layer.check(x, k, act, b)
    # a second call on the used workspace gives the same bits
    first = b["y"].clone()
    layer.call(gpu(x, layer.t), k, act, b)
    assert torch.equal(first, b["y"])


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
def test_every_token_on_the_same_experts(w):
    """64 rows on one expert (the most there can be), none on the others."""
    rng = np.random.default_rng(4)
    layer = Layer(rng, w, 6, 128, 192)
    layer.b_gate = np.array([0, 30, 0, 0, 20, 0], np.float32)
    layer.gb = gpu(layer.b_gate)
    x = as_type(rng.standard_normal((64, 128)), w)
    for k in (1, 2):
        b = layer.buffers(64, k)
        layer.call(gpu(x, layer.t), k, "gelu", b)
        layer.check(x, k, "gelu", b)
        assert (b["idx"].cpu().numpy() == [1, 4][:k]).all()


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
def test_masked_experts_and_tokens_without_numbers(w):
    """Experts switched off by a bias of minus infinity are never chosen; a
    token with a NaN or an infinity leaves the other tokens alone; a mask that
    leaves nothing gives NaN outputs and valid experts, as softmax does."""
    import torch
    rng = np.random.default_rng(6)
    layer = Layer(rng, w, 5, 128, 320)
    layer.b_gate = np.array([0, -np.inf, 0, -np.inf, 0], np.float32)
    layer.gb = gpu(layer.b_gate)
    x = as_type(rng.standard_normal((11, 128)), w)
    x[3, 7] = np.nan
    x[8, 100] = np.inf
    good = [t for t in range(11) if t not in (3, 8)]
    b = layer.buffers(11, 2)
    layer.call(gpu(x, layer.t), 2, "silu", b)
    clean = x.copy()
    clean[[3, 8]] = 0.0
    layer.check(clean, 2, "silu", b, rows=good)
    idx = b["idx"].cpu().numpy()
    assert not np.isin(idx[good], (1, 3)).any()
    assert ((idx >= 0) & (idx < 5)).all() and (idx[:, 0] != idx[:, 1]).all()
    y = b["y"].double().cpu().numpy()
    assert np.isnan(y[3]).all() and not np.isfinite(y[8]).any()
    # two experts left for k = 2, then one, then none
    for left in (2, 1, 0):
        layer.b_gate = np.where(np.arange(5) < left, 0.0, -np.inf).astype(np.float32)
        layer.gb = gpu(layer.b_gate)
        b = layer.buffers(11, 2)
        layer.call(gpu(clean, layer.t), 2, "silu", b)
        idx = b["idx"].cpu().numpy()
        assert ((idx >= 0) & (idx < 5)).all() and (idx[:, 0] != idx[:, 1]).all()
        y = b["y"].double().cpu().numpy()
        if left == 0:
            assert np.isnan(y).all()
        else:
            assert np.isfinite(y).all()
        if left == 1:
            assert (idx[:, 0] == 0).all() and (b["gate"].cpu().numpy() == [1.0, 0.0]).all()


def test_a_token_does_not_depend_on_its_neighbours():
    """Output bits of a token alone and in a batch of 64."""
    import torch
    rng = np.random.default_rng(12)
    for w in ("bf16", "mx4"):
        layer = Layer(rng, w, 3, 256, 256)
        x = as_type(rng.standard_normal((64, 256)), w)
        b = layer.buffers(64, 2)
        layer.call(gpu(x, layer.t), 2, "gelu", b)
        for t in (0, 31, 63):
            one = layer.buffers(1, 2)
            layer.call(gpu(x[t:t + 1], layer.t), 2, "gelu", one)
            assert np.array_equal(one["idx"].cpu().numpy()[0], b["idx"].cpu().numpy()[t])
            assert np.array_equal(one["y"][0].float().cpu().numpy(), b["y"][t].float().cpu().numpy())


def test_choices_and_gates_match_luffy_route():
    """Experts and gates are luffy_route's, near-ties included."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(21)
    T, E, d = 64, 16, 256
    for w in ("f32", "bf16"):
        layer = Layer(rng, w, E, d, 64)
        layer.w_gate[5] = layer.w_gate[2]                      # equal logits: the lower index
        layer.gg = gpu(layer.w_gate, layer.t)
        layer.b_gate[5] = layer.b_gate[2]
        layer.gb = gpu(layer.b_gate)
        x = gpu(as_type(rng.standard_normal((T, d)), w), layer.t)
        for k in (1, 2):
            b = layer.buffers(T, k)
            layer.call(x, k, "gelu", b)
            o = dict(idx=torch.empty_like(b["idx"]), gate=torch.empty_like(b["gate"]),
                     pos=torch.empty_like(b["idx"]), perm=torch.empty(T * k, dtype=torch.int32, device="cuda"),
                     off=torch.empty(E + 1, dtype=torch.int32, device="cuda"))
            ws = torch.empty(max(256, L.route_workspace_size(T, E, k)), dtype=torch.uint8, device="cuda")
            L.luffy_route(x, layer.gg, layer.gb, k, 0.0, o["idx"], o["gate"], o["pos"], o["perm"], o["off"], ws)
            assert torch.equal(o["idx"], b["idx"])
            assert (o["gate"] - b["gate"]).abs().max().item() <= 2e-6


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
def test_graph_replays_and_another_stream(w):
    """Captured once and replayed on new tokens, with eager calls between, and
    eager calls on a side stream: the same bits."""
    import torch
    rng = np.random.default_rng(2)
    layer = Layer(rng, w, 4, 128, 256)
    T, k = 12, 2
    x = torch.empty(T, 128, dtype=layer.t, device="cuda").normal_()
    b, other = layer.buffers(T, k), layer.buffers(T, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.call(x, k, "gelu", b)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.call(x, k, "gelu", b)
    for _ in range(4):
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        layer.call(x, k, "gelu", other, stream=side)
        side.synchronize()
        assert torch.equal(b["y"], other["y"]) and torch.equal(b["idx"], other["idx"])
