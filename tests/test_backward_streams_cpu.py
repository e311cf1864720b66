"""The buffers that a layer's or a block's first backward makes belong to the stream that
the backward runs on, and those that a change of type replaces are held until the stream
that wrote them is done (allocations and streams are watched: no GPU needed)."""
import contextlib
import os

import pytest


@pytest.fixture(scope="module", autouse=True)
def lib():
    import paper_2411_15419_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2411_15419_amd import build
        build.build()
    return L.load_library()


@pytest.fixture
def watch(monkeypatch):
    """made: (stream that is current, bytes) of every allocation; held: (tensor, stream)."""
    import torch
    import paper_2411_15419_amd as L
    for name in ("luffy_block_norm", "luffy_block_norm_backward", "luffy_route_scored", "luffy_route_scored_backward",
                 "luffy_condense", "luffy_expert_ffn_keep", "luffy_expert_ffn_backward_kept", "luffy_combine_many",
                 "luffy_combine_many_backward", "luffy_combine_backward", "luffy_expert_ffn_backward",
                 "luffy_mx8_quantize", "luffy_mx8_dequantize"):
        monkeypatch.setattr(L, name, lambda *a, **kw: None)
    current, made, held = ["current"], [], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def empty(*a, **kw):
        t = real(*a, **kw)
        made.append((current[-1], t.data_ptr()))
        return t

    real = torch.empty
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(L, "_stream", lambda stream: stream or "current")
    monkeypatch.setattr(L, "_hold", lambda t, raw: held.append((t.data_ptr(), raw)), raising=False)
    return made, held


def layers():
    import torch
    import paper_2411_15419_amd as L
    bf = dict(dtype=torch.bfloat16)
    w = lambda: (torch.zeros(4, 64, **bf), torch.zeros(4), torch.zeros(4, 64, 64, **bf), torch.zeros(4, 64, 64, **bf))  # noqa: E731
    kw = dict(k=2, act="gelu", threshold=0.9, T=8)
    return dict(layer=L.MoELayer(*w(), **kw), block=L.MoEBlock(*w(), w_pre=torch.ones(64), gate=torch.ones(64), **kw),
                sharing=L.MoEBlock(*w(), w_pre=torch.ones(64), shares=L.MoEBlock(*w(), w_pre=torch.ones(64), keep8=True,
                                                                                  **kw), **kw))


@pytest.mark.parametrize("which", ["layer", "block", "sharing"])
def test_buffers_of_the_stream_that_uses_them(watch, which):
    import torch
    made, held = watch
    x = torch.zeros(8, 64, dtype=torch.bfloat16)
    f = layers()[which]
    if which != "layer":
        f(x)
    del made[:]
    f.backward(x, x, "side")
    assert made and {s for s, _ in made} == {"side"}
    old = {f._bwd[n].data_ptr() for n in ("dw1", "dw2")}
    del made[:]
    f.backward(x, x, "side")                           # nothing new
    assert not made and not held
    f.backward(x, x, "other", torch.bfloat16)          # another type: those two and no more
    assert len(made) == 2 and {s for s, _ in made} == {"other"}
    assert {p for p, _ in held} == old and {s for _, s in held} == {"side"}
    assert f._bwd["dw1"].dtype == f._bwd["dw2"].dtype == torch.bfloat16
    del made[:], held[:]
    f.backward(x, x, None, torch.float32)
    assert {s for s, _ in made} == {"current"} and {s for _, s in held} == {"other"}
