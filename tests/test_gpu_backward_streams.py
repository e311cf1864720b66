"""A layer's and a block's whole step on a stream of its own, with a change of the weight
gradients' type: the bits of the same step on the current stream."""
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


T, d, E, k, d_ff = 200, 128, 4, 2, 192


def make(block):
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(1)
    t = lambda *s: torch.from_numpy(rng.standard_normal(s) / np.sqrt(s[-1])).to(torch.bfloat16).cuda()  # noqa: E731
    w = t(E, d), torch.zeros(E, device="cuda"), t(E, d_ff, d), t(E, d, d_ff)
    kw = dict(k=k, act="gelu", threshold=2.0, T=T)     # (no two tokens alike: every sum has a fixed order)
    return L.MoEBlock(*w, w_pre=torch.ones(d, device="cuda"), **kw) if block else L.MoELayer(*w, **kw)


def tensors(out):
    return [t for o in out for t in (o.values() if isinstance(o, dict) else [o])]


@pytest.mark.parametrize("block", [False, True])
def test_a_step_on_a_stream(block):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(T, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    types = (torch.float32, torch.bfloat16, torch.float32)
    here, there = make(block), make(block)
    y = here(x)
    want = [y.clone()]
    for dt in types:
        out = tensors(here.backward(x, dy, None, dt))
        rows = int(here.buf.rep_offsets[-1])           # (a layer's dx_rep: the rows in use)
        want += [t[:rows].clone() if t.shape == (T * k, d) else t.clone() for t in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [there(x, s)]
    with torch.cuda.stream(s):
        got = [got[0].clone()]
        for dt in types:
            out = tensors(there.backward(x, dy, s, dt))
            got += [t[:rows].clone() if t.shape == (T * k, d) else t.clone() for t in out]
            junk = [torch.full((E, d_ff, d), 7.0, device="cuda", dtype=dt) for _ in range(2)]
            del junk
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
