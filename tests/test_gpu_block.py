"""Whole blocks on the GPU, forward and backward: norm, scored router,
condensation, experts with 8-bit kept activations, combine, norm, gate and
residual, against the 64-bit form with the GPU's decisions."""
import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu

# In the 2-norm, relative: a block's results go through six bf16 roundings on the
# way there (u, act(Z), y_rep, y, o, the output itself) and nine on the way back (those
# that matter of the six, dy, dy_rep, dZ, dx_rep, du, dx), at most 2^-8 each, so 15 /
# 256 = 6 %; Z's 8 bits are off by at most m / 128 (m: the largest of 32, about 2.5
# of their root mean square), uniformly, 1.2 % of Z, and as much for the kept u.
# Each is an independent error; added up they stay below
NORM = 0.085


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def tensor(a, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()


def numpy(t):
    return None if t is None else t.double().cpu().numpy()


def make(seed, T, d, E, k, d_ff, *, norm="rms", gate="channel", bias=False, act="gelu", threshold=2.0, **kw):
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(seed)
    vec = lambda at: tensor(at + 0.1 * rng.standard_normal(d))  # noqa: E731
    w = dict(w_gate=tensor(rng.standard_normal((E, d)) / np.sqrt(d), "bf16"), b_gate=tensor(0.1 * rng.standard_normal(E)),
             w1=tensor(rng.standard_normal((E, d_ff, d)) / np.sqrt(d), "bf16"),
             w2=tensor(rng.standard_normal((E, d, d_ff)) / np.sqrt(d_ff), "bf16"))
    around = dict(w_pre=vec(1.0), b_pre=vec(0.0) if bias else None, w_post=vec(1.0), b_post=vec(0.0) if bias else None,
                  gate={"channel": vec(0.5), "token": tensor(rng.uniform(0.2, 1, (T, d)), "bf16"), "none": None}[gate])
    return L.MoEBlock(**w, **around, k=k, act=act, threshold=threshold, T=T, norm=norm, **kw)


def stream(seed, T, d, centres=None):
    rng = np.random.default_rng(seed)
    if centres:
        c = rng.standard_normal((centres, d))
        return tensor(c[rng.integers(0, centres, T)] + 0.05 * rng.standard_normal((T, d)), "bf16")
    return tensor(rng.standard_normal((T, d)), "bf16")


def reference(block, x, dout, dlogits=None):
    b = block.buf
    dec = {n: getattr(b, n).cpu().numpy().astype(np.int64) for n in ("slot_pos", "rep_row", "rep_of_pos", "rep_token",
                                                                     "rep_offsets")}
    dec["idx"] = b.topk_idx.cpu().numpy().astype(np.int64)
    dec["rep_token"] = dec["rep_token"][: dec["rep_offsets"][-1]]
    p = dict(x=numpy(x), w_gate=numpy(block.w_gate), b_gate=numpy(block.b_gate), w1=numpy(block.w1), w2=numpy(block.w2),
             w_pre=numpy(block.w_pre), b_pre=numpy(block.b_pre), w_post=numpy(block.w_post), b_post=numpy(block.b_post),
             gate=numpy(block.gate))
    cfg = dict(norm=block.norm, eps=block.eps, res_scale=block.res_scale, score=block.score,
               renormalise=block.renormalise, scale=block.scale, act=block.act)
    o, s = B.block_forward(p, dec, cfg)
    return o, B.block_backward(p, dec, cfg, s, dout, dlogits), dec


def far(got, ref):
    return np.linalg.norm(numpy(got) - ref) / np.linalg.norm(ref)


CASES = {
    "sigmoid groups": dict(T=200, d=256, E=16, k=4, d_ff=320, score="sigmoid", groups=4, top_groups=2, group_best=2,
                           scale=2.0, capacity_factor=1.1),
    "softmax layer norm": dict(T=131, d=192, E=8, k=2, d_ff=512, norm="layer", bias=True, gate="token", act="silu",
                               renormalise=False, keep8=False),
    "eight of many": dict(T=150, d=128, E=48, k=8, d_ff=128, score="sigmoid", gate="none", res_scale=0.7),
    "one expert a token": dict(T=97, d=128, E=4, k=1, d_ff=256, renormalise=False),
}


@pytest.mark.parametrize("name", CASES)
def test_block(name):
    kw = dict(CASES[name])
    T, d = kw["T"], kw["d"]
    if kw.get("score") == "sigmoid":
        kw["balance"] = tensor(0.05 * np.random.default_rng(3).standard_normal(kw["E"]))
    block = make(1, **kw)
    x = stream(2, T, d)
    rng = np.random.default_rng(4)
    dout = tensor(rng.standard_normal((T, d)), "bf16")
    dl = tensor(0.1 * rng.standard_normal((T, kw["E"])))
    o = block(x).clone()
    dx, g = block.backward(x, dout, dlogits=dl)
    ref_o, ref, _ = reference(block, x, numpy(dout), numpy(dl))
    assert far(o, ref_o) < NORM
    assert far(dx, ref["dx"]) < NORM
    assert set(g) == {n for n in ref if n != "dx" and (n not in ("db_pre", "db_post") or block.b_pre is not None)}
    for n, v in g.items():
        assert far(v, ref[n]) < NORM, n
    again, _ = block.backward(x, dout, dlogits=dl)     # from what was kept, once more
    assert far(again, ref["dx"]) < NORM


def test_condensed_block():
    """Similar tokens: a representative's gradient reaches its own row alone."""
    block = make(5, 512, 256, 8, 2, 256, score="sigmoid", threshold=0.9)
    x = stream(6, 512, 256, centres=40)
    dout = tensor(np.random.default_rng(7).standard_normal((512, 256)), "bf16")
    o = block(x).clone()
    dx, g = block.backward(x, dout)
    ref_o, ref, dec = reference(block, x, numpy(dout))
    assert 0 < dec["rep_offsets"][-1] < 512          # of 1024 slots
    assert far(o, ref_o) < NORM and far(dx, ref["dx"]) < NORM
    for n, v in g.items():
        assert far(v, ref[n]) < NORM, n


def test_chained_blocks():
    """Two blocks of which the first's last pass is the second's first: as two blocks
    by themselves."""
    import torch
    kw = dict(T=160, d=256, E=8, k=3, d_ff=256, score="sigmoid", norm="layer", bias=True)
    a, b = make(8, **kw), make(9, **kw)
    x, dout = stream(10, 160, 256), stream(11, 160, 256)
    o1 = a(x).clone()
    o2 = b(o1).clone()
    d1, g2 = b.backward(o1, dout)
    d1, g2 = d1.clone(), {n: v.clone() for n, v in g2.items()}
    dx, g1 = a.backward(x, d1)
    dx, g1 = dx.clone(), {n: v.clone() for n, v in g1.items()}
    # chained: the same bits forward
    p1 = a(x, following=b)
    p2 = b(p1, normed=True)
    assert torch.equal(o1, p1) and torch.equal(o2, p2)
    ds, h2 = b.backward(p1, dout)
    ex, h1 = a.backward(x, ds, following=b)
    # the stream's gradient between them is rounded before the norm's share is added
    # instead of after: some more roundings of 2^-8
    assert far(ex, numpy(dx)) < 4 * 2.0 ** -8
    for n in g1:
        assert far(h1[n], numpy(g1[n])) < 4 * 2.0 ** -8, n
    for n in g2:
        assert far(h2[n], numpy(g2[n])) < 4 * 2.0 ** -8, n


def test_blocks_with_history():
    """The first of a stack computes every pair: the plain block's bits.  The second
    condenses with the first's record."""
    import torch
    kw = dict(T=512, d=256, E=8, k=2, d_ff=256, score="sigmoid", threshold=0.9)
    plain, a, b = make(15, **kw), make(15, **kw, history=(0.2, 0.95)), make(16, **kw, history=(0.2, 0.95))
    x = stream(17, 512, 256, centres=40)
    dout = tensor(np.random.default_rng(18).standard_normal((512, 256)), "bf16")
    want, o1 = plain(x), a(x)
    assert torch.equal(want, o1) and torch.equal(plain.buf.rep_of_pos, a.buf.rep_of_pos)
    o1 = o1.clone()
    o2 = b(o1, hist_in=a.record).clone()
    dx, g = b.backward(o1, dout)
    ref_o, ref, dec = reference(b, o1, numpy(dout))
    assert 0 < dec["rep_offsets"][-1] < 1024
    assert far(o2, ref_o) < NORM and far(dx, ref["dx"]) < NORM
    for n, v in g.items():
        assert far(v, ref[n]) < NORM, n


def test_captured_block():
    """Forward and backward in a graph, replayed on other inputs beside eager work."""
    import torch
    block = make(12, 300, 256, 16, 4, 256, score="sigmoid", groups=4, top_groups=2, threshold=0.9, capacity_factor=1.0)
    x, dout = stream(13, 300, 256, centres=60), stream(14, 300, 256)
    block(x)
    block.backward(x, dout)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = block(x)
        dx, g = block.backward(x, dout)
    for seed in (1, 2, 3):
        x.copy_(stream(seed, 300, 256, centres=60))
        graph.replay()
        got = [t.clone() for t in (o, dx, *g.values())]
        idx = block.buf.topk_idx.clone()
        o2 = block(x).clone()
        dx2, g2 = block.backward(x, dout)
        torch.cuda.synchronize()
        assert torch.equal(idx, block.buf.topk_idx) and torch.equal(got[0], o2)
        for a, b in zip(got[1:], (dx2, *g2.values())):
            # (the order in which a group's members are added is not fixed)
            assert float((a.double() - b.double()).norm() / b.double().norm()) < 2.0 ** -6


@pytest.mark.parametrize("k", [1, 2, 3, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_combine_many(k, dtype):
    """Against the sum in 64 bits, and its transpose."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(k)
    T, d, E = 77, 320, 9
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    slot_pos, perm, off = B.buckets(idx, E, 0.8)
    S = len(perm)
    rep = rng.random(S) < 0.5
    rep[off[:-1][off[:-1] < S]] = True
    rep_of = np.maximum.accumulate(np.where(rep, np.arange(S), -1))
    row = (np.cumsum(rep) - 1)[rep_of]
    R = int(rep.sum())
    i32 = lambda a, n: torch.from_numpy(np.concatenate([a, np.full(n - len(a), 10 ** 9)]).astype(np.int32)).cuda()  # noqa: E731
    sp = torch.from_numpy(slot_pos.astype(np.int32)).cuda()
    rr, pt = i32(row, T * k), i32(perm, T * k)
    o32, ro = i32(off, E + 1), i32(np.concatenate([[0], np.cumsum(rep)])[off], E + 1)
    y_rep = tensor(rng.standard_normal((T * k, d)), dtype)
    gate, dy = tensor(rng.uniform(0, 1, (T, k))), tensor(rng.standard_normal((T, d)), dtype)
    y = torch.empty_like(dy)
    L.luffy_combine_many(y_rep, rr, sp, gate, y)
    n = numpy(y_rep), numpy(gate), numpy(dy)
    kept = slot_pos >= 0
    at = np.where(kept, row[np.maximum(slot_pos, 0)], 0)
    terms = np.where(kept, n[1], 0.0)[..., None] * n[0][at]
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    bound = 8 * 2.0 ** -24 * np.abs(terms).sum(1) + 1.01 * half * np.abs(terms.sum(1))
    assert (np.abs(numpy(y) - terms.sum(1)) <= bound).all()
    if k <= 2:
        z = torch.empty_like(y)
        L.luffy_combine(y_rep, rr, sp, gate, z)
        assert torch.equal(y, z)
    dy_rep, dgate = torch.full_like(y_rep, -9.0), torch.empty_like(gate)
    ws = torch.empty(L.combine_backward_workspace_size(T, k, T * k), dtype=torch.uint8, device="cuda")
    L.luffy_combine_many_backward(dy, y_rep, rr, pt, sp, gate, o32, ro, dy_rep, dgate, ws)
    ref, size = np.zeros((R, d)), np.zeros((R, d))
    for j in range(k):
        m = kept[:, j]
        np.add.at(ref, at[m, j], (n[1][:, j, None] * n[2])[m])
        np.add.at(size, at[m, j], np.abs(n[1][:, j, None] * n[2])[m])
    got = numpy(dy_rep)
    assert (np.abs(got[:R] - ref) <= T * 2.0 ** -24 * size + 1.01 * half * np.abs(ref)).all()
    assert (got[R:] == -9.0).all()
    dots = (n[2][:, None] * n[0][at])
    ref = np.where(kept, dots.sum(2), 0.0)
    assert (np.abs(numpy(dgate) - ref) <= d * 2.0 ** -24 * np.abs(dots).sum(2)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_condense_with_many_choices(dtype):
    """luffy_condense on buckets of six choices a token, against the oracle."""
    import torch
    import paper_2411_15419_amd as L
    from oracle import luffy_oracle as O
    rng = np.random.default_rng(20)
    T, d, E, k = 300, 128, 12, 6
    c = rng.standard_normal((30, d))
    x = tensor(c[rng.integers(0, 30, T)] + 0.03 * rng.standard_normal((T, d)), dtype)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    slot_pos, perm, off = B.buckets(idx, E, 1.0)
    cap = L.capacity(T, k, E, 1.0)
    i32 = lambda n: torch.full((n,), -5, dtype=torch.int32, device="cuda")  # noqa: E731
    pt = i32(T * k)
    pt[:len(perm)] = torch.from_numpy(perm.astype(np.int32)).cuda()
    o32 = torch.from_numpy(off.astype(np.int32)).cuda()
    of, row, ro, tok, deg = i32(T * k), i32(T * k), i32(E + 1), i32(T * k), i32(T * k)
    ws = torch.empty(L.condense_workspace_size(T, d, E, k, cap), dtype=torch.uint8, device="cuda")
    L.luffy_condense(x, pt, o32, k, cap, 0.9, of, row, ro, tok, None, deg, ws)
    ref = O.condense(numpy(x), perm, off, 0.9)
    S = len(perm)
    assert np.array_equal(of[:S].cpu().numpy(), np.asarray(ref.rep_of_pos)[:S])
    assert np.array_equal(ro.cpu().numpy(), ref.rep_offsets)
    R = int(ro[-1])
    assert 0 < R < S
    assert np.array_equal(row[:S].cpu().numpy(), np.asarray(ref.rep_row)[:S])
    assert np.array_equal(tok[:R].cpu().numpy(), np.asarray(ref.rep_token)[:R])


@pytest.mark.parametrize("T,k,R,rows", [(1, 1, 1, 20000), (2048, 3, 4095, 4095), (2048, 3, 4096, 4096), (3000, 4, 4097, 9000),
                                        (5000, 5, 8192, 8192), (5000, 8, 20001, 40000), (3, 2, 0, 5000)])
def test_combine_many_backward_of_many_representatives(T, k, R, rows):
    """More representatives than a block counts, numbers around its edges, and room for
    more rows than there are slots."""
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(R)
    S, d = T * k if R else 0, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    slot_pos = torch.randperm(T * k, generator=gen, device="cuda").to(torch.int32).view(T, k) if R else torch.full((T, k), -1, **i32)
    tok = torch.zeros(T * k, **i32)
    if R:
        tok[slot_pos.flatten().long()] = torch.arange(T, **i32).repeat_interleave(k)
    rep_row = torch.cat([torch.arange(R, **i32), torch.randint(0, max(R, 1), (T * k - R,), generator=gen, **i32)])
    off, ro = torch.tensor([0, S], **i32), torch.tensor([0, R], **i32)
    dy, gate = torch.randn(T, d, generator=gen, device="cuda"), torch.rand(T, k, generator=gen, device="cuda")
    y_rep = torch.randn(rows, d, generator=gen, device="cuda")
    dy_rep, dgate = torch.full_like(y_rep, -9.0), torch.empty_like(gate)
    ws = torch.empty(L.combine_backward_workspace_size(T, k, rows), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        L.luffy_combine_many_backward(dy, y_rep, rep_row, tok, slot_pos, gate, off, ro, dy_rep, dgate, ws)
    assert bool((dy_rep[R:] == -9.0).all())
    if not R:
        assert not bool(dgate.any())
        return
    at = rep_row[slot_pos.long()].long()
    terms = gate.double()[..., None] * dy.double()[:, None]
    want = torch.zeros(R, d, dtype=torch.float64, device="cuda").index_add_(0, at.flatten(), terms.view(-1, d))
    size = torch.zeros_like(want).index_add_(0, at.flatten(), terms.abs().view(-1, d))
    most = int(torch.bincount(at.flatten()).max())
    assert bool(((dy_rep[:R].double() - want).abs() <= (most + 1) * 2.0 ** -24 * size).all())
    dots = dy.double()[:, None] * y_rep.double()[at]
    assert bool(((dgate.double() - dots.sum(2)).abs() <= d * 2.0 ** -24 * dots.abs().sum(2)).all())
