"""Microscaled products with several tiles a block: the next tile's first stages
are fetched under the epilogue of the one before, whose results turn in the
same LDS.  A block has a second tile from 513 tiles on (two blocks a CU)."""
import numpy as np
import pytest

from oracle import mx4_oracle as M

pytestmark = pytest.mark.gpu

PLACES = 2 * 256     # blocks of such a product at most


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def matrix(gen, groups, rows, cols):
    """Any codes, blocks of scales from 1/4 to 4: (values, scales, float64 values)."""
    import torch
    import paper_2411_15419_amd as L
    q = torch.randint(0, 256, (groups, rows, cols // 2), dtype=torch.uint8, device="cuda", generator=gen)
    s = torch.randint(125, 130, (groups, (cols + 255) // 256, rows, 8), dtype=torch.uint8, device="cuda", generator=gen)
    s.view(groups, -1, rows, 8)[:, -1, :, (cols // 32 - 1) % 8 + 1:] = 0
    v = torch.empty(groups, rows, cols, device="cuda")
    L.luffy_mx4_dequantize(q, s, v)
    return q, s, v


def rows_of(kind, rng):
    """Rows of the experts, several of them without any: (list, narrow tiles?)."""
    if kind == "narrow":          # at most 64 rows an expert on average
        n = rng.integers(1, 130, 48)
        n[[3, 17, 18, 47]] = 0
        n[5], n[9] = 64, 65
        while n.sum() > 64 * 48:
            n[n.argmax()] //= 2
        return [int(v) for v in n], 64
    return [1100, 0, 130, 1, 2300, 128, 700], 128


@pytest.mark.parametrize("K", [96, 256, 512, 544, 768, 1312])     # 1, 1, 2, 3, 3 and 6 stages
@pytest.mark.parametrize("kind,out", [("narrow", "f32"), ("narrow", "bf16"), ("wide", "f32"), ("wide", "bf16")])
def test_matmul(kind, out, K):
    """Every result exact: the sums' magnitudes stay below 2^24 of their step."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(K)
    gen = torch.Generator(device="cuda").manual_seed(K)
    n, bn = rows_of(kind, rng)
    E, R, N = len(n), sum(n), 4064
    assert (R <= 64 * E) == (kind == "narrow")
    tiles = sum(-(-v // bn) for v in n) * (-(-N // 128))
    assert tiles > 2 * PLACES
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    (xq, xs, xv), (wq, ws, wv) = matrix(gen, 1, R + 5, K), matrix(gen, E, N, K)
    t = torch.float32 if out == "f32" else torch.bfloat16
    y = torch.full((R + 5, N), 768.0, dtype=t, device="cuda")
    L.luffy_mx4_matmul(xq[0], xs[0], torch.from_numpy(off).cuda(), wq, ws, y)
    assert (y[R:] == 768.0).all()
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        x, w = xv[0, a:b].double(), wv[e].double()
        assert (x.abs() @ w.abs().t()).max().item() < 2.0 ** (24 - 6)     # values are multiples of 1/8 each
        assert torch.equal(y[a:b], (x @ w.t()).to(t)), e


@pytest.mark.parametrize("kind", ["narrow", "wide"])
@pytest.mark.parametrize("act,d", [("gelu", 128), ("silu", 512), ("gelu", 704), ("silu", 1344)])
def test_expert_ffn(kind, act, d):
    """Each row the same bits as in calls of a hundred rows of one expert, whose
    products have one tile a block; those are compared with the 64-bit form
    elsewhere."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(d)
    gen = torch.Generator(device="cuda").manual_seed(d)
    n, bn = rows_of(kind, rng)
    E, R, d_ff = len(n), sum(n), 4160
    assert (R <= 64 * E) == (kind == "narrow")
    assert sum(-(-v // bn) for v in n) * (-(-d_ff // 128)) > 2 * PLACES
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    x = normal(R, d).to(torch.bfloat16)
    (w1, s1), (w2, s2) = L.mx4_weights(0.1 * normal(E, d_ff, d)), L.mx4_weights(0.1 * normal(E, d, d_ff))

    def call(x, off, *w):
        rows, experts = x.shape[0], w[0].shape[0]
        y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(L.mx4_expert_ffn_workspace_size(rows, experts, d, d_ff), dtype=torch.uint8, device="cuda")
        L.luffy_mx4_expert_ffn(x, None, torch.tensor(off, dtype=torch.int32, device="cuda"), *w, act, rows, y, ws)
        return y
    y = call(x, off, w1, s1, w2, s2)
    assert torch.isfinite(y).all()
    for e in range(E):
        part = [t[e:e + 1].contiguous() for t in (w1, s1, w2, s2)]
        for a in range(int(off[e]), int(off[e + 1]), 100):
            b = min(a + 100, int(off[e + 1]))
            assert torch.equal(y[a:b], call(x[a:b].contiguous(), [0, b - a], *part)), (e, a)
