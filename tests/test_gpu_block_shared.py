"""MoEBlocks that share what they work with, on the GPU: the bits of blocks by
themselves."""
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


T, d, E, k, d_ff = 160, 256, 8, 3, 320


def tensor(a, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()


def make(seed, **kw):
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(seed)
    vec = lambda at: tensor(at + 0.1 * rng.standard_normal(d))  # noqa: E731
    return L.MoEBlock(tensor(rng.standard_normal((E, d)) / np.sqrt(d), "bf16"), tensor(0.1 * rng.standard_normal(E)),
                      tensor(rng.standard_normal((E, d_ff, d)) / np.sqrt(d), "bf16"),
                      tensor(rng.standard_normal((E, d, d_ff)) / np.sqrt(d_ff), "bf16"), w_pre=vec(1.0), w_post=vec(1.0),
                      gate=vec(0.5), k=k, act="silu", threshold=2.0, T=T, score="sigmoid", **kw)


def stream(seed):
    return tensor(np.random.default_rng(seed).standard_normal((T, d)), "bf16")


def step(blocks, x, dout, chained):
    """Outputs and gradients of blocks one after the other (no two tokens alike: every
    sum has a fixed order)."""
    xs = [x]
    for i, b in enumerate(blocks):
        more = dict(following=blocks[i + 1] if i + 1 < len(blocks) else None, normed=i > 0) if chained else {}
        xs.append(b(xs[-1], **more).clone())
    out = []
    for i in reversed(range(len(blocks))):
        more = dict(following=blocks[i + 1] if i + 1 < len(blocks) else None) if chained else {}
        dout, g = blocks[i].backward(xs[i], dout, **more)
        out += g.values()       # (dw_pre of a chained block: from the one before it)
    return xs[1:] + [t.clone() for t in out + [dout]]


@pytest.mark.parametrize("chained", [False, True])
def test_shared_blocks(chained):
    import torch
    apart = [make(i, keep8=True) for i in range(3)]
    first = make(0, keep8=True)
    shared = [first, make(1, shares=first), make(2, shares=first)]
    for seed in (1, 2):
        x, dout = stream(seed), stream(seed + 10)
        want, got = step(apart, x, dout, chained), step(shared, x, dout, chained)
        assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_shared_blocks_captured():
    import torch
    first = make(0, keep8=True)
    shared = [first, make(1, shares=first)]
    x, dout = stream(1), stream(2)
    step(shared, x, dout, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(shared, x, dout, True)
    for seed in (3, 4, 5):
        x.copy_(stream(seed))
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in got]
        want = step(shared, x, dout, True)
        assert all(torch.equal(a, b) for a, b in zip(have, want))


def test_a_block_alone_takes_u_as_it_is():
    """Nothing is rounded where u stays: dW1 and dW_gate of the u that the experts had."""
    import torch
    block, rounded = make(5), make(5, keep8=True)
    x, dout = stream(6), stream(7)
    o, o8 = block(x).clone(), rounded(x).clone()
    u = block.u.clone()
    dx, g = block.backward(x, dout)
    assert torch.equal(o, o8) and torch.equal(block.u, u)
    _, g8 = rounded.backward(x, dout)
    assert torch.equal(g["dw2"], g8["dw2"]) and not torch.equal(g["dw1"], g8["dw1"])
    # u in 8 bits is off by up to 2^-7 of a block's largest value
    assert float((g["dw1"] - g8["dw1"]).norm() / g["dw1"].norm()) < 2.0 ** -6
