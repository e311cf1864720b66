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


def test_rows_past_4_gib():
    """Values, scales, rows and results whose offsets pass 32 bits: the last rows
    are what they are on their own."""
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, cols = 2 ** 18 + 37, 32768          # q just past 4 GiB, bf16 values past 16
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    q = torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(cols // 256, rows, 8, dtype=torch.uint8, device="cuda")
    L.luffy_mx4_quantize(x, q, s)
    tail = x[-41:].clone()
    tq, ts = torch.empty_like(q[-41:]), torch.empty(cols // 256, 41, 8, dtype=torch.uint8, device="cuda")
    L.luffy_mx4_quantize(tail, tq, ts)
    assert torch.equal(q[-41:], tq) and torch.equal(s[:, -41:], ts)
    L.luffy_mx4_dequantize(q, s, x)
    back = torch.empty_like(tail)
    L.luffy_mx4_dequantize(tq, ts, back)
    assert torch.equal(x[-41:], back)
    del x
    wq, ws = L.mx4_weights(torch.empty(1, 64, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen))
    y, ty = torch.empty(rows, 64, device="cuda"), torch.empty(41, 64, device="cuda")
    L.luffy_mx4_matmul(q, s, None, wq, ws, y)
    L.luffy_mx4_matmul(tq, ts, None, wq, ws, ty)
    v = torch.empty(1, 64, cols, device="cuda")
    L.luffy_mx4_dequantize(wq, ws, v)
    # 32768 float32 additions in some order
    bound = 32768 * 2.0 ** -24 * (back.double().abs() @ v[0].double().abs().t())
    for got in (ty, y[-41:]):
        assert ((got.double() - back.double() @ v[0].double().t()).abs() <= bound).all()


@pytest.mark.parametrize("w,E,d,d_ff", [("bf16", 64, 4096, 11008), ("mx4", 9, 32768, 32768)])
def test_experts_past_4_gib(w, E, d, d_ff):
    """The last expert's weights lie past 4 GiB; the same weights as the first
    expert give the same bits."""
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(4)
    if w == "bf16":
        w1, w2 = (torch.empty(E, *m, dtype=torch.bfloat16, device="cuda").normal_(0, 0.02, generator=gen)
                  for m in ((d_ff, d), (d, d_ff)))
        scales = [None, None]
        tensors = [w1, w2]
    else:
        w1, w2 = (torch.randint(0, 256, (E, a, b // 2), dtype=torch.uint8, device="cuda", generator=gen)
                  for a, b in ((d_ff, d), (d, d_ff)))
        scales = [torch.randint(112, 120, (E, b // 256, a, 8), dtype=torch.uint8, device="cuda", generator=gen)
                  for a, b in ((d_ff, d), (d, d_ff))]
        tensors = [w1, w2] + scales
    assert (E - 1) * w1[0].numel() * w1.element_size() >= 2 ** 32
    w_gate = torch.zeros(E, d, dtype=torch.bfloat16, device="cuda")
    for T in (1, 9):
        x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        out = []
        for e in (E - 1, 0):
            if e == 0:
                for t in tensors:
                    t[0].copy_(t[E - 1])
            b_gate = torch.full((E,), -50.0, device="cuda")
            b_gate[e] = 50.0
            idx, gate = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
            y = torch.empty_like(x)
            ws = torch.empty(L.moe_few_workspace_size(T, d, E, 1, d_ff), dtype=torch.uint8, device="cuda")
            L.luffy_moe_few(x, w_gate, b_gate, w1, w2, 1, "gelu", idx, gate, y, ws, w1_scale=scales[0],
                            w2_scale=scales[1])
            assert (idx == e).all()
            out.append(y)
        assert torch.isfinite(out[0]).all() and out[0].abs().max() > 0
        assert torch.equal(out[0], out[1])
        tensors[0][0].zero_()
