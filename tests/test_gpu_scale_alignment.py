"""Scales of 4-bit matrices at 8-byte aligned addresses that are not 16-byte
aligned, which the contract allows: the same bits as from aligned ones."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def at_eight(t):
    """The same tensor eight bytes into an allocation of its own."""
    import torch
    raw = torch.zeros(t.numel() + 16, dtype=torch.uint8, device=t.device)
    out = raw[8:8 + t.numel()].view(t.shape)
    out.copy_(t)
    assert out.data_ptr() % 16 == 8
    return out


@pytest.mark.parametrize("T", [1, 7, 40])
def test_step(T):
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(T)
    E, k, d, d_ff = 5, 2, 320, 576
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)
    x, w_gate = normal(T, d), normal(E, d)
    (w1, s1), (w2, s2) = L.mx4_weights(normal(E, d_ff, d)), L.mx4_weights(normal(E, d, d_ff))
    out = []
    for a, b in ((s1, s2), (at_eight(s1), at_eight(s2))):
        idx, gate = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
        y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(L.moe_few_workspace_size(T, d, E, k, d_ff), dtype=torch.uint8, device="cuda")
        L.luffy_moe_few(x, w_gate, None, w1, w2, k, "silu", idx, gate, y, ws, w1_scale=a, w2_scale=b)
        out.append(y)
    assert torch.isfinite(out[0]).all() and torch.equal(out[0], out[1])


def test_quantise_and_product():
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(37, 544, generator=gen, device="cuda")
    wq, ws = L.mx4_weights(torch.randn(1, 96, 544, generator=gen, device="cuda"))
    q = torch.empty(37, 272, dtype=torch.uint8, device="cuda")
    s = torch.empty(3, 37, 8, dtype=torch.uint8, device="cuda")
    y, z = torch.empty(37, 96, device="cuda"), torch.empty(37, 96, device="cuda")
    L.luffy_mx4_quantize(x, q, s)
    L.luffy_mx4_matmul(q, s, None, wq, ws, y)
    t = at_eight(torch.zeros_like(s))
    L.luffy_mx4_quantize(x, q, t)
    assert torch.equal(s, t)
    L.luffy_mx4_matmul(q, t, None, wq, at_eight(ws), z)
    assert torch.equal(y, z)
    back, again = torch.empty_like(x), torch.empty_like(x)
    L.luffy_mx4_dequantize(q, s, back)
    L.luffy_mx4_dequantize(q, t, again)
    assert torch.equal(back, again)
