"""What a MoEBlock holds between its call and its backward, byte for byte, alone and where
blocks share what they work with (buffers alone: no GPU needed)."""
import dataclasses
import os

import pytest


@pytest.fixture(scope="module", autouse=True)
def lib():
    import paper_2411_15419_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2411_15419_amd import build
        build.build()
    return L.load_library()


T, d, E, k, d_ff = 96, 128, 6, 3, 320


def make(**kw):
    import torch
    import paper_2411_15419_amd as L
    bf = dict(dtype=torch.bfloat16)
    size = dict(T=T, k=k, d=d, d_ff=d_ff, E=E)
    size.update({n: kw.pop(n) for n in list(kw) if n in size})
    T_, k_, d_, f_, E_ = (size[n] for n in ("T", "k", "d", "d_ff", "E"))
    return L.MoEBlock(torch.zeros(E_, d_, **bf), torch.zeros(E_), torch.zeros(E_, f_, d_, **bf), torch.zeros(E_, d_, f_, **bf),
                      w_pre=torch.ones(d_), w_post=torch.ones(d_), k=k_, act="gelu", threshold=0.9, T=T_, **kw)


def storages(block, weights=("w_gate", "b_gate", "w1", "w2", "w_pre", "w_post")):
    """Bytes of every storage that a block holds, its weights left out."""
    import torch
    found, seen = {}, [v for n, v in vars(block).items() if n not in weights]
    while seen:
        v = seen.pop()
        if isinstance(v, torch.Tensor):
            found[v.untyped_storage().data_ptr()] = v.untyped_storage().nbytes()
        elif isinstance(v, dict):
            seen += v.values()
        elif dataclasses.is_dataclass(v):
            seen += vars(v).values()
    return found


def kept(keep8):
    S, groups = T * k, lambda n: (n + 255) // 256
    b = S * d_ff + groups(d_ff) * S * 8 + 2 * S * d + 2 * 2 * T * d + 4 * T * E      # Z, y_rep, y and o, logits
    b += 4 * (8 * S + T + 2 * (E + 1))       # the choices and the condensation
    return b + (T * d + groups(d) * T * 8 if keep8 else 2 * T * d)


def working(block):
    b = block.buf
    return 2 * T * d + sum(w.numel() for w in (b.ws_route, b.ws_condense, b.ws_ffn))


def test_a_block_alone_keeps_u_once():
    block = make()
    assert not block.keep8 and not hasattr(block, "uq")
    assert sum(storages(block).values()) == kept(False) + working(block) - 2 * T * d


def test_blocks_that_share_keep_no_more_than_they_say():
    import torch
    first = make(keep8=True)
    others = [make(shares=first), make(shares=first)]
    others.append(make(shares=others[-1]))                     # through another: the same buffers
    assert sum(storages(first).values()) == kept(True) + working(first)
    base = storages(first)
    for b in others:
        assert b.keep8 and b.u is first.u
        own = {p: n for p, n in storages(b).items() if p not in base}
        assert sum(own.values()) == kept(True)
    # the backward: dx, the stream's gradient and the weights' are a block's own
    grads = 2 * (2 * T * d) + 4 * E * d + 4 * E + 2 * (4 * E * d * d_ff) + 2 * 4 * d
    for b in [others[0], first, others[1]]:                    # (any may be the first)
        b._gradients(torch.float32)
    base = storages(first)
    for b in others[:2]:
        own = {p: n for p, n in storages(b).items() if p not in base}
        assert sum(own.values()) == kept(True) + grads


def test_what_cannot_be_shared_is_refused():
    import paper_2411_15419_amd as L
    first = make(keep8=True)
    with pytest.raises(L.LuffyError, match="keep u in 8 bits"):
        make(shares=make())
    with pytest.raises(L.LuffyError, match="keep u in 8 bits"):
        make(shares=first, keep8=False)
    for other in (dict(T=T + 1), dict(k=2), dict(d=192), dict(d_ff=256), dict(E=8), dict(capacity_factor=0.5)):
        with pytest.raises(L.LuffyError, match="same sizes"):
            make(shares=first, **other)
    with pytest.raises(L.LuffyError, match="same sizes"):
        make(k=2, shares=make(k=2, keep8=True), history=(0.1, 0.9))
