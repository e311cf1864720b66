"""Calls of chained MoEBlocks in an order in which one would read what another has written
over are refused.  The library's calls are left out: no GPU needed."""
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
def make(monkeypatch):
    import torch
    import paper_2411_15419_amd as L
    for name in ("luffy_block_norm", "luffy_block_norm_backward", "luffy_route_scored", "luffy_route_scored_backward",
                 "luffy_condense", "luffy_expert_ffn_keep", "luffy_expert_ffn_backward_kept", "luffy_combine_many",
                 "luffy_combine_many_backward", "luffy_mx8_quantize", "luffy_mx8_dequantize"):
        monkeypatch.setattr(L, name, lambda *a, **kw: None)
    bf = dict(dtype=torch.bfloat16)

    def block(**kw):
        return L.MoEBlock(torch.zeros(4, 64, **bf), torch.zeros(4), torch.zeros(4, 64, 64, **bf),
                          torch.zeros(4, 64, 64, **bf), w_pre=torch.ones(64), k=2, act="gelu", threshold=0.9, T=8, **kw)
    return block


@pytest.fixture
def x():
    import torch
    return torch.zeros(8, 64, dtype=torch.bfloat16)


def refused(match):
    import paper_2411_15419_amd as L
    return pytest.raises(L.LuffyError, match=match)


KINDS = [dict(), dict(keep8=True)]


@pytest.mark.parametrize("kind", KINDS + ["shared"], ids=str)
def test_orders_that_hold(make, x, kind):
    if kind == "shared":
        a = make(keep8=True)
        b, c = make(shares=a), make(shares=a)
    else:
        a, b, c = (make(**kind) for _ in range(3))
    for _ in range(2):
        c(b(a(x, following=b), normed=True, following=c), normed=True)
        c.backward(x, x)
        c.backward(x, x)                               # once more, from what is kept
        b.backward(x, x, following=c)
        a.backward(x, x, following=b)
        if kind != "shared":
            a.backward(x, x, following=b)
        a(x)
        b(x)
        b.backward(x, x)
        a.backward(x, x)
    a(x, following=b)
    b(x, normed=True)
    if kind != "shared":
        b(x, normed=True)                              # of the same u
    b.backward(x, x)
    a.backward(x, x, following=b)


@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_a_backward_of_another_call(make, x, kind):
    """The following block's backward is of the call before the last one."""
    a, b = make(**kind), make(**kind)
    a(x, following=b)
    b(x, normed=True)
    b.backward(x, x)
    a(x, following=b)
    with refused("comes first"):
        a.backward(x, x, following=b)
    b(x, normed=True)
    with refused("comes first"):
        a.backward(x, x, following=b)
    b.backward(x, x)
    a.backward(x, x, following=b)
    # a block that was called by itself in between, or behind another one
    other = make(**kind)
    other(x, following=b)
    b(x, normed=True)
    b.backward(x, x)
    with refused("comes first"):
        a.backward(x, x, following=b)
    other.backward(x, x, following=b)


def test_no_u_to_start_from(make, x):
    a, b = make(keep8=True), make(keep8=True)
    with refused("normed"):
        b(x, normed=True)                              # nothing has written it
    a(x, following=b)
    b(x, normed=True)
    b.backward(x, x)
    with refused("normed"):
        b(x, normed=True)                              # it is that of the 8 bits now
    b(x)
    with refused("normed"):
        b(x, normed=True)                              # and now its own
    a(x, following=b)
    b(x, normed=True)


def test_a_u_that_was_written_over(make, x):
    """Without 8 bits the next call's u is in the place of the one that a backward needs."""
    a, b = make(), make()
    a(x, following=b)
    b(x, normed=True)
    a(x, following=b)
    with refused("written over"):
        b.backward(x, x)
    b(x, normed=True)
    b.backward(x, x)
    a, b = make(keep8=True), make(keep8=True)          # with them it is not needed
    a(x, following=b)
    b(x, normed=True)
    a(x, following=b)
    b.backward(x, x)


def test_what_sharing_blocks_write_over(make, x):
    a = make(keep8=True)
    b, c = make(shares=a), make(shares=a)
    a(x, following=b)
    c(x)                                               # its u in the place of b's
    with refused("normed"):
        b(x, normed=True)
    a(x, following=b)
    b(x, normed=True)
    c(x)
    b.backward(x, x)
    c.backward(x, x)                                   # its du in the place of b's
    with refused("written over"):
        a.backward(x, x, following=b)
    b.backward(x, x)
    a.backward(x, x, following=b)
    with refused("written over"):
        a.backward(x, x, following=b)                  # its own du is
