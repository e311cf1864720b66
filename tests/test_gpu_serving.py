"""A layer that serves (ServingLayer): prompts through the condensed layer on
4-bit weights, decoding steps through luffy_moe_few; and the forms that the
products choose between by size."""
import numpy as np
import pytest

from oracle import mx4_oracle as M
from test_gpu_few import Layer, as_type, gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def weights(rng, E, d, d_ff, dtype):
    return [gpu(m.astype(np.float32), dtype) for m in
            (0.1 * rng.standard_normal((E, d)), 0.05 * rng.standard_normal((E, d_ff, d)),
             0.05 * rng.standard_normal((E, d, d_ff)))]


@pytest.mark.parametrize("k,act,gather", [(1, "silu", False), (2, "gelu", True)])
def test_prompt_and_steps(k, act, gather):
    """Half the prompt repeats the other half, so half its rows condense: the
    representatives' rows are those of luffy_mx4_expert_ffn on the quantised
    weights, a repeated token has its representative's output, and every token's
    y is the gate-weighted sum.  Steps are luffy_moe_few's."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(20 + k)
    E, d, d_ff, T = 5, 256, 320, 300
    w_gate, w1, w2 = weights(rng, E, d, d_ff, torch.bfloat16)
    layer = L.ServingLayer(w_gate, None, w1, w2, k=k, act=act, threshold=0.99, T=T, gather_x_rep=gather)
    half = rng.standard_normal((T // 2, d)).astype(np.float32)
    x = gpu(np.concatenate([half, half]), torch.bfloat16)
    y = layer(x).clone()
    b = layer.buf
    R = int(b.rep_offsets[-1])
    assert R == T * k // 2
    assert torch.equal(y[:T // 2], y[T // 2:])
    q1, s1 = L.mx4_weights(w1)
    q2, s2 = L.mx4_weights(w2)
    rep = torch.empty_like(b.y_rep)
    ws = torch.empty(L.mx4_expert_ffn_workspace_size(T * k, E, d, d_ff), dtype=torch.uint8, device="cuda")
    L.luffy_mx4_expert_ffn(x, b.rep_token, b.rep_offsets, q1, s1, q2, s2, act, T * k, rep, ws)
    assert torch.equal(rep[:R], b.y_rep[:R])
    row = torch.gather(b.rep_row.long(), 0, b.slot_pos.reshape(-1).long())
    want = (rep[row].double().reshape(T, k, d) * b.topk_gate.double()[..., None]).sum(1)
    # k products and their sum in float32, rounded to bf16
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -22 * (rep[row].double().reshape(T, k, d).abs()).sum(1)
    assert ((y.double() - want).abs() <= bound).all()
    for n in (1, 3, 64):
        xs = x[:n].contiguous()
        idx, gate = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
        z = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(L.moe_few_workspace_size(n, d, E, k, d_ff), dtype=torch.uint8, device="cuda")
        L.luffy_moe_few(xs, w_gate, None, q1, q2, k, act, idx, gate, z, ws, w1_scale=s1, w2_scale=s2)
        assert torch.equal(layer.step(xs), z)
        assert torch.equal(layer.step_idx[:n], idx) and torch.equal(layer.step_gate[:n], gate)
        assert torch.equal(idx, b.topk_idx[:n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_plain_weights(dtype):
    """microscaled=False: the prompt is MoELayer's, steps are the 64-bit layer's."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(31)
    lay = Layer(rng, dtype, 4, 128, 192)
    args = dict(k=2, act="gelu", threshold=0.9, T=100)
    x = as_type(rng.standard_normal((100, 128)), dtype)
    serve = L.ServingLayer(lay.gg, lay.gb, lay.g1, lay.g2, microscaled=False, **args)
    plain = L.MoELayer(lay.gg, lay.gb, lay.g1, lay.g2, **args)
    assert torch.equal(serve(gpu(x, lay.t)), plain(gpu(x, lay.t)))
    y = serve.step(gpu(x[:11], lay.t))
    lay.check(x[:11], 2, "gelu", dict(idx=serve.step_idx[:11], gate=serve.step_gate[:11], y=y))


def test_refusals():
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(1)
    args = dict(k=1, act="gelu", threshold=0.9, T=8)
    w_gate, w1, w2 = weights(rng, 2, 64, 64, torch.float32)
    with pytest.raises(L.LuffyError, match="bf16 activations"):
        L.ServingLayer(w_gate, None, w1, w2, **args)
    layer = L.ServingLayer(w_gate, None, w1, w2, microscaled=False, **args)
    with pytest.raises(L.LuffyError, match="no backward"):
        layer.backward(None, None)
    for n in (0, 65):
        with pytest.raises(L.LuffyError, match="1 to 64"):
            layer.step(torch.zeros(n, 64, device="cuda"))
    with pytest.raises(L.LuffyError):
        layer.step(torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("w", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("k", [1, 2])
def test_forms_agree(w, k):
    """Up to eight slots (tokens times choices) run without LDS columns.  The
    same tokens in every batch on both sides of that: each against the 64-bit
    layer; a token's bits do not depend on the others while the rows of a work
    item are the same (one wave's part of K as far as an eighth)."""
    import torch
    rng = np.random.default_rng(40 + k)
    layer = Layer(rng, w, 4, 320, 448)
    x = as_type(rng.standard_normal((11, 320)), w)
    first = None
    for T in (1, 2, 3, 4, 5, 8, 9, 11):
        b = layer.buffers(T, k)
        layer.call(gpu(x[:T], layer.t), k, "silu", b)
        layer.check(x[:T], k, "silu", b)
        if first is None:
            first = b["y"].clone()
        assert torch.equal(first, b["y"][:1]), T


def test_forms_agree_on_one_expert_for_all():
    """Every slot on the same one or two experts, the others idle."""
    import torch
    rng = np.random.default_rng(50)
    layer = Layer(rng, "bf16", 6, 192, 256, bias=False)
    layer.b_gate = np.array([-90, 0, -90, 30, -90, -90], np.float32)
    layer.gb = gpu(layer.b_gate)
    x = as_type(rng.standard_normal((9, 192)), "bf16")
    for T, k in ((4, 2), (8, 1), (9, 1), (5, 2)):
        b = layer.buffers(T, k)
        layer.call(gpu(x[:T], layer.t), k, "gelu", b)
        layer.check(x[:T], k, "gelu", b)


@pytest.mark.parametrize("rows", [
    [1500],                     # 12 row tiles by 8 column tiles: more than a block of tiles each way
    [0, 97, 700, 1, 0, 1300],   # wide tiles, experts without rows and with one
    [3, 0, 96, 64, 65, 1]])     # narrow tiles
def test_matmul_over_many_tiles(rows):
    """Small integers, so that every sum is exact in float32."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(len(rows) + rows[0])
    E, R, N, K = len(rows), sum(rows), 992, 544
    code = lambda r: rng.integers(0, 16, (r, K)).astype(np.uint8)
    scale = lambda r: rng.integers(127, 129, (r, K // 32)).astype(np.uint8)
    xc, xs = code(R), scale(R)
    wc, ws = [code(N) for _ in rows], [scale(N) for _ in rows]
    xq, xsc = M.pack(xc, xs)
    wq, wsc = map(np.stack, zip(*[M.pack(c, s) for c, s in zip(wc, ws)]))
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    y = torch.full((R, N), -7.0, device="cuda")
    L.luffy_mx4_matmul(gpu(xq), gpu(xsc), gpu(off) if E > 1 else None, gpu(wq), gpu(wsc), y)
    xv = M.values(xc, xs)
    want = np.concatenate([xv[a:b] @ M.values(c, s).T for a, b, c, s in zip(off[:-1], off[1:], wc, ws)])
    assert np.array_equal(y.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,N", [(4001, 3840), (3900, 4064)])
def test_one_matrix_that_fills_the_cus(dtype, R, N):
    """Sizes of the largest tiles (about 16 by 16 of them, the last ones ragged);
    small integers, exact in float32 (and their sums' nearest bf16)."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(R)
    K = 2144
    xc, wc = (rng.integers(0, 16, (r, K)).astype(np.uint8) for r in (R, N))
    xs, ws = (rng.integers(127, 129, (r, K // 32)).astype(np.uint8) for r in (R, N))
    (xq, xsc), (wq, wsc) = M.pack(xc, xs), M.pack(wc, ws)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    y = torch.full((R, N), -7.0, dtype=t, device="cuda")
    L.luffy_mx4_matmul(gpu(xq), gpu(xsc), None, gpu(wq[None]), gpu(wsc[None]), y)
    want = torch.from_numpy(M.values(xc, xs)).cuda() @ torch.from_numpy(M.values(wc, ws)).cuda().t()
    assert torch.equal(y, want.to(t))
