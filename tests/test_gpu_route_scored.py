"""The scored router on the GPU against its 64-bit form: choices, gates and
buckets, and its gradients."""
import itertools

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {"f32": U32, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def tensor(a, dtype="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to({"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32}[dtype]).cuda()


def numpy(t):
    return t.double().cpu().numpy()


class Router:
    """Inputs, and a call's outputs with their numpy forms."""

    def __init__(self, seed, dtype, T, d, E, k, score="sigmoid", balance=True, groups=1, top_groups=1, group_best=1,
                 renorm=True, scale=1.0, cf=0.0, spread=None):
        rng = np.random.default_rng(seed)
        self.dtype, self.T, self.d, self.E, self.k, self.score, self.cf = dtype, T, d, E, k, score, cf
        self.kw = dict(groups=groups, top_groups=top_groups, group_best=group_best)
        self.renorm, self.scale = renorm, scale
        self.x = tensor(rng.standard_normal((T, d)), dtype)
        self.w = tensor((spread or 1.0 / np.sqrt(d)) * rng.standard_normal((E, d)), dtype)
        self.b = tensor(0.1 * rng.standard_normal(E))
        self.bal = tensor((0.05 if score == "sigmoid" else 0.5 / E) * rng.standard_normal(E)) if balance else None

    def run(self, stream=None, out=None):
        import torch
        import paper_2411_15419_amd as L
        T, E, k = self.T, self.E, self.k
        i32 = dict(dtype=torch.int32, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        out = out or dict(topk_idx=torch.full((T, k), -7, **i32), topk_gate=torch.full((T, k), -7.0, **f32),
                          logits=torch.full((T, E), -7.0, **f32), slot_pos=torch.full((T, k), -7, **i32),
                          perm_token=torch.full((T * k,), -7, **i32), offsets=torch.full((E + 1,), -7, **i32),
                          workspace=torch.empty(L.route_workspace_size(T, E, k), dtype=torch.uint8, device="cuda"),
                          inv_norm=torch.full((T,), -7.0, **f32))
        L.luffy_route_scored(self.x, self.w, self.b, k, self.score, self.cf, balance=self.bal, renormalise=self.renorm,
                             scale=self.scale, stream=stream, **out, **self.kw)
        return out

    def logits64(self):
        return numpy(self.x) @ numpy(self.w).T + numpy(self.b)

    def check(self, out, exact_gates=True):
        l = self.logits64()
        bal = None if self.bal is None else numpy(self.bal)
        idx = B.choose(l, self.k, self.score, bal, **self.kw)
        got = out["topk_idx"].cpu().numpy()
        assert np.array_equal(got, idx), np.argwhere(got != idx)[:4].tolist()
        slot_pos, perm, offsets = B.buckets(idx, self.E, self.cf)
        assert np.array_equal(out["offsets"].cpu().numpy(), offsets)
        assert np.array_equal(out["slot_pos"].cpu().numpy(), slot_pos)
        perm_got = out["perm_token"].cpu().numpy()
        assert np.array_equal(perm_got[:len(perm)], perm) and (perm_got[len(perm):] == -7).all()
        # a logit: at most d / 4 + 20 roundings of the sum of |x w| (<= |x| |w|), and its last one
        n = np.linalg.norm(numpy(self.x), axis=1)
        wn = np.linalg.norm(numpy(self.w), axis=1)
        dl = (self.d / 4 + 20) * U32 * (n[:, None] * wn + np.abs(numpy(self.b))) + U32 * np.abs(l)
        assert (np.abs(numpy(out["logits"]) - l) <= dl).all()
        # a gate: relative to itself by twice the logits' error (its own and the others'),
        # and 2^-20 + |l| 2^-22 for exponentials and divisions
        g = B.gates(l, idx, self.score, self.renorm, self.scale)
        rel = 2 * dl.max(1, keepdims=True) + 2.0 ** -20 + np.abs(l).max(1, keepdims=True) * 2.0 ** -22
        assert (np.abs(numpy(out["topk_gate"]) - g) <= rel * np.abs(g)).all()
        inv = 1.0 / np.maximum(n, 1e-300)
        inv[n == 0] = 0.0
        assert (np.abs(numpy(out["inv_norm"]) - inv) <= self.d * U32 * inv).all()
        return idx


CASES = [  # dtype, T, d, E, k, score, balance, groups, top, best, renorm, cf
    ("bf16", 1, 64, 1, 1, "softmax", False, 1, 1, 1, False, 0.0),
    ("bf16", 1, 1024, 16, 2, "softmax", False, 1, 1, 1, True, 0.0),
    ("bf16", 17, 256, 13, 3, "sigmoid", True, 1, 1, 1, True, 0.0),
    ("f32", 33, 320, 8, 8, "softmax", True, 1, 1, 1, False, 1.1),
    ("bf16", 130, 512, 64, 8, "sigmoid", True, 8, 4, 2, True, 1.0),
    ("f32", 130, 192, 64, 8, "sigmoid", False, 8, 3, 2, True, 0.0),
    ("bf16", 200, 128, 32, 4, "softmax", True, 16, 5, 1, True, 1.25),
    ("bf16", 65, 2112, 24, 6, "sigmoid", True, 8, 2, 2, False, 0.0),
    ("f32", 64, 64, 48, 5, "softmax", False, 3, 1, 1, False, 0.7),
    ("bf16", 1000, 64, 64, 8, "sigmoid", True, 16, 2, 2, True, 1.0),
    ("bf16", 300, 320, 6, 1, "sigmoid", False, 3, 2, 1, False, 0.5),
    ("bf16", 257, 1088, 64, 7, "softmax", True, 2, 1, 2, True, 0.0),
    ("bf16", 90, 4096, 8, 2, "softmax", False, 4, 4, 2, True, 0.0),
    ("f32", 77, 4096, 64, 8, "softmax", True, 64, 64, 1, True, 0.0),
    ("bf16", 16, 1088, 64, 8, "sigmoid", True, 8, 4, 2, True, 1.0),      # one block and one launch up to 16 tokens
    ("f32", 16, 320, 40, 6, "softmax", True, 10, 3, 2, True, 0.0),
    ("bf16", 7, 2112, 24, 4, "softmax", False, 1, 1, 1, False, 0.6),
    ("f32", 2, 64, 16, 3, "sigmoid", False, 4, 2, 2, False, 0.0),
    ("bf16", 15, 4096, 12, 2, "softmax", True, 3, 1, 1, True, 0.0),
    ("f32", 9, 128, 64, 8, "sigmoid", True, 1, 1, 1, True, 0.5),
    ("bf16", 17, 1088, 64, 8, "sigmoid", True, 8, 4, 2, True, 1.0),      # one block, two launches
    ("bf16", 32, 256, 33, 8, "softmax", True, 3, 2, 2, True, 0.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_route(case):
    dtype, T, d, E, k, score, bal, groups, top, best, renorm, cf = case
    r = Router(T + E, dtype, T, d, E, k, score, bal, groups, top, best, renorm, 2.5 if renorm else 1.0, cf)
    r.check(r.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score,bal,groups", [("softmax", False, 1), ("softmax", True, 4), ("sigmoid", True, 4),
                                               ("sigmoid", False, 4)])
def test_close_calls(dtype, score, bal, groups):
    """Experts whose weights differ in the last bits of a few values, and twins:
    gaps down to nothing, where float32 sums cannot tell."""
    r = Router(3, dtype, 256, 512, 32, 6, score, bal, groups, max(1, groups // 2), 2)
    w = numpy(r.w)
    w[1::2] = w[0::2]                                  # twins
    rng = np.random.default_rng(4)
    for e in range(3, 32, 4):                          # and near twins: one value, by one step or two
        c = rng.integers(0, 512)
        w[e, c] *= 1.0 + (2.0 ** -6 if dtype == "bf16" else 2.0 ** -20)
    r.w = tensor(w, dtype)
    r.b = tensor(np.repeat(np.random.default_rng(5).standard_normal(16) * 0.1, 2))
    if bal:
        r.bal = tensor(np.repeat(np.random.default_rng(6).standard_normal(16) * 0.02, 2))
    r.check(r.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [5, 300])
def test_groups_that_turn(dtype, T):
    """Float32 sums tie two groups, the exact ones keep the other: it has fewer good
    experts, and those that take their places are near to none of the first choice."""
    r = Router(31, dtype, T, 2048, 16, 4, "softmax", False, 4, 2, 1)
    x, w = np.zeros((T, 2048)), np.zeros((16, 2048))
    x[:, 0], x[:, 128], x[:, 256], x[:, 300] = 64, 1, 64, 1
    w[:, 0], w[:, 256] = 16, -16                          # 1024 - 1024
    w[4:8, 128] = 2.0 ** -15                              # lost beside 1024 in float32
    w[:, 300] = [5, 4, 3, 2, 5, -1, -2, -3, 6, 1.5, 0.5, 0.25, -5, -6, -7, -8]
    x[::3, 300] = 0.5                                     # the same at another scale
    r.x, r.w, r.b = tensor(x, dtype), tensor(w, dtype), tensor(np.zeros(16))
    idx = r.check(r.run())
    assert (idx == [8, 4, 9, 10]).all()
    w[10], w[9] = w[9], 0                                 # now 8's group has a tie as well: 9 and 10
    w[9, 300], w[9, 128] = 1.5, 2.0 ** -15
    w[10, 0], w[10, 256], w[9, 0], w[9, 256] = 16, -16, 16, -16
    r.w = tensor(w, dtype)
    idx = r.check(r.run())
    assert (idx[1::3] == [8, 4, 9, 10]).all()
    w[[9, 10]] = w[[10, 9]]
    r.w = tensor(w, dtype)
    idx = r.check(r.run())
    assert (idx[1::3] == [8, 4, 10, 9]).all()


@pytest.mark.parametrize("E", [16, 48])
def test_a_token_alone_or_among_others(E):
    """The choices, buckets and logits' bits of 16 tokens are those of one call for
    each: the largest call in one launch, and the same rows in a larger one."""
    import torch
    r = Router(33, "bf16", 40, 1088, E, 4, "sigmoid", True, 8, 4, 2)
    want = r.run()
    x = r.x
    for lo, hi in ((0, 16), (16, 17), (17, 31)):
        r.x, r.T = x[lo:hi], hi - lo
        out = r.run()
        r.check(out)
        for n in ("topk_idx", "logits", "topk_gate"):
            assert torch.equal(out[n], want[n][lo:hi]), n


def test_cancelling_rows():
    """Sums of large products that cancel: the logits are small beside |x| |w|."""
    r = Router(8, "bf16", 192, 1024, 16, 4, "sigmoid", True)
    x, w = numpy(r.x) * 100, numpy(r.w)
    x[:, 512:] = -x[:, :512]
    w[:, 512:] = w[:, :512] * (1 + 2.0 ** -7 * (np.random.default_rng(2).random((16, 512)) < 0.05))
    r.x, r.w = tensor(x, "bf16"), tensor(w, "bf16")
    r.check(r.run())


def test_zero_rows_and_no_bias():
    r = Router(9, "bf16", 40, 128, 12, 3, "softmax", False)
    r.x[::3] = 0
    r.b = tensor(np.zeros(12))
    out = r.run()
    r.check(out)
    assert out["topk_idx"][0].tolist() == [0, 1, 2]


def test_numbers_that_are_none():
    """NaN and infinities in a row: experts within range, each once, and the other
    rows as ever."""
    r = Router(10, "bf16", 64, 256, 32, 8, "sigmoid", True, 8, 2, 2)
    clean = r.run()
    r.x[5, 7], r.x[9, 0], r.x[11] = float("nan"), float("inf"), float("-inf")
    out = r.run()
    keep = [t for t in range(64) if t not in (5, 9, 11)]
    for name in ("topk_idx", "topk_gate", "logits"):
        assert bool((out[name][keep] == clean[name][keep]).all())
    for t in (5, 9, 11):
        e = out["topk_idx"][t].tolist()
        assert len(set(e)) == 8 and min(e) >= 0 and max(e) < 32
    assert out["topk_idx"][5].tolist() == list(range(8))     # nothing is a number: the lowest of the lowest groups
    r = Router(10, "f32", 64, 256, 32, 8, "softmax", False)
    r.w[3, 3] = float("nan")                                  # one expert has no logits at all
    idx = r.run()["topk_idx"]
    assert not bool((idx == 3).any())


@pytest.mark.parametrize("T,d,E", [(33000, 128, 64), (9000, 192, 24), (66000, 64, 12)])
def test_numbers_that_are_none_among_many(T, d, E):
    """The same in the larger calls' kernels, and an expert whose weights are none: it is
    chosen by no token, the other choices are those of a call without it."""
    import torch
    r = Router(34, "bf16", T, d, E, 4, "sigmoid", True, 4, 2, 2)
    clean = r.run()
    bad = [0, 17, T // 2, T - 1]
    r.x[bad[0], 7], r.x[bad[1], 0], r.x[bad[2]], r.x[bad[3], d - 1] = (float("nan"), float("inf"), float("-inf"),
                                                                        float("nan"))
    out = r.run()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[bad] = False
    for name in ("topk_idx", "topk_gate", "logits"):
        assert bool((out[name][keep] == clean[name][keep]).all())
    chosen = out["topk_idx"][bad].long()
    assert bool(((chosen >= 0) & (chosen < E)).all())
    assert all(len(set(row)) == 4 for row in chosen.tolist())
    counts = torch.bincount(out["topk_idx"].flatten().long(), minlength=E)
    assert torch.equal(torch.diff(out["offsets"].long()), counts)
    r = Router(35, "bf16", T, d, E, 3, "softmax", False)
    r.w[5, 3] = float("nan")
    idx = r.run()["topk_idx"].long()
    l = r.x.double() @ torch.nan_to_num(r.w.double()).t() + r.b.double()
    l[:, 5] = -torch.inf
    assert torch.equal(idx, torch.sort(l, dim=1, descending=True, stable=True).indices[:, :3])


def test_masked_experts():
    """balance -infinity: chosen only where nothing else is left."""
    r = Router(12, "bf16", 50, 128, 16, 4, "sigmoid", True, 4, 2, 2)
    bal = numpy(r.bal)
    bal[:8] = -np.inf                       # two whole groups
    bal[8:14] = -np.inf                     # of the others two experts are left
    r.bal = tensor(bal)
    out = r.run()
    idx = out["topk_idx"].cpu().numpy()
    ref = B.choose(r.logits64(), 4, "sigmoid", bal, groups=4, top_groups=2, group_best=2)
    assert np.array_equal(idx, ref)
    assert (np.sort(idx[:, :2], 1) == [14, 15]).all()


def test_huge_values():
    """Rows whose float32 sums leave the type's range are decided in float64."""
    r = Router(13, "f32", 24, 128, 8, 2, "softmax", False)
    r.x *= 1e25
    r.w *= 1e20
    out = r.run()
    assert np.array_equal(out["topk_idx"].cpu().numpy(), B.choose(r.logits64(), 2, "softmax"))


@pytest.mark.parametrize("dtype,T,d,E,k", [("bf16", 20011, 256, 16, 4), ("bf16", 33000, 128, 64, 8),
                                            ("f32", 9001, 64, 24, 3), ("bf16", 16400, 1088, 60, 2),
                                            ("bf16", 40003, 2048, 32, 4), ("bf16", 17003, 64, 40, 5),
                                            ("bf16", 66000, 320, 45, 8)])
def test_many_tokens(dtype, T, d, E, k):
    """Every kernel size; the choices against a stable sort of 64-bit scores."""
    import torch
    r = Router(T, dtype, T, d, E, k, "sigmoid", True)
    out = r.run()
    l = r.x.double() @ r.w.double().t() + r.b.double()
    c = torch.sigmoid(l) + r.bal.double()
    idx = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(out["topk_idx"].long(), idx)
    flat = idx.t().reshape(-1)
    order = torch.sort(flat, stable=True).indices
    assert torch.equal(out["perm_token"].long(), order % T)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(T * k, device="cuda")
    assert torch.equal(out["slot_pos"].long(), pos.view(k, T).t())
    g = torch.sigmoid(l).gather(1, idx)
    g = g / g.sum(1, keepdim=True)
    assert float(((out["topk_gate"].double() - g).abs() / g).max()) < 1e-5 * (1 + d / 1024)


def test_runs_repeat_and_streams():
    """Two calls on streams of their own, with workspaces of their own, and again."""
    import torch
    a = Router(21, "bf16", 3000, 512, 32, 4, "sigmoid", True, 8, 4, 2, cf=1.1)
    b = Router(22, "bf16", 2000, 256, 64, 8, "softmax", False)
    ra, rb = a.run(), b.run()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    again = []
    for _ in range(3):
        for r, s in ((a, streams[0]), (b, streams[1])):
            with torch.cuda.stream(s):
                again.append((ra if r is a else rb, r.run()))
    torch.cuda.synchronize()
    for want, got in again:
        assert all(torch.equal(want[n], got[n]) for n in want if n != "workspace")


def test_captured():
    """A captured call replayed on other inputs, eager work in between."""
    import torch
    r = Router(23, "bf16", 700, 512, 32, 4, "sigmoid", True, 8, 4, 2, cf=1.0)
    out = r.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.run(out=out)
    for seed in (1, 2, 3):
        r.x.copy_(tensor(np.random.default_rng(seed).standard_normal((700, 512)), "bf16"))
        graph.replay()
        want = r.run()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n][: int(want["offsets"][-1])], out[n][: int(want["offsets"][-1])])
                   for n in ("topk_idx", "topk_gate", "logits", "slot_pos", "perm_token", "offsets"))


# ---------------------------------------------------------------- gradients
class Gradients:
    def __init__(self, seed, dtype, T, d, E, k, score, renorm, extra, reps, capacity=False, scale=1.5):
        import torch
        rng = np.random.default_rng(seed)
        self.a = dict(score=score, renorm=renorm, scale=scale)
        self.dtype, self.T, self.d, self.E, self.k = dtype, T, d, E, k
        self.x, self.w = tensor(rng.standard_normal((T, d)), dtype), tensor(rng.standard_normal((E, d)), dtype)
        self.l = tensor(2 * rng.standard_normal((T, E)))
        idx = B.choose(numpy(self.l), k, score)
        slot_pos, _, off = B.buckets(idx, E, 0.8 if capacity else 0.0)
        S = int(off[-1])
        dg = np.where(slot_pos >= 0, rng.standard_normal((T, k)), 0.0)
        self.idx, self.dg = tensor(idx, "i32"), tensor(dg)
        self.extra = tensor(0.1 * rng.standard_normal((T, E))) if extra else None
        self.rep = {}
        if reps:
            rep = rng.random(S) < 0.6
            rep[off[:-1][off[:-1] < S]] = True
            rep_of = np.maximum.accumulate(np.where(rep, np.arange(S), -1))
            row = (np.cumsum(rep) - 1)[rep_of]
            fill = np.full(T * k - S, 10 ** 9)         # never read: behind the last position
            self.rep = dict(dx_rep=tensor(rng.standard_normal((int(rep.sum()) + 1, d)), dtype),
                            slot_pos=tensor(slot_pos, "i32"),
                            rep_of_pos=tensor(np.concatenate([rep_of, fill]), "i32"),
                            rep_row=tensor(np.concatenate([row, fill]), "i32"))
            self.rep["dx_rep"][-1] = float("nan")       # a row in no use
        self.torch = torch

    def run(self, out=None):
        import paper_2411_15419_amd as L
        t = self.torch
        out = out or dict(dx=t.full_like(self.x, float("nan")),
                          dw_gate=t.full((self.E, self.d), float("nan"), device="cuda"),
                          db_gate=t.full((self.E,), float("nan"), device="cuda"),
                          workspace=t.empty(L.route_scored_backward_workspace_size(self.T, self.d, self.E),
                                            dtype=t.uint8, device="cuda"))
        L.luffy_route_scored_backward(self.x, self.w, self.a["score"], self.l, self.idx, self.dg, **out,
                                      renormalise=self.a["renorm"], scale=self.a["scale"], dlogits=self.extra,
                                      **self.rep)
        return out

    def check(self, out):
        n = lambda v: None if v is None else numpy(v)  # noqa: E731
        rep = {m: n(v) for m, v in self.rep.items()}
        for m in ("slot_pos", "rep_of_pos", "rep_row"):
            if m in rep:
                rep[m] = rep[m].astype(np.int64)
        a = (self.a["score"], self.a["renorm"], self.a["scale"])
        l, idx = n(self.l), self.idx.cpu().numpy().astype(np.int64)
        dx, dw, db = B.route_backward(n(self.x), n(self.w), l, idx, n(self.dg), *a, n(self.extra), **rep)
        # dl: at most 64 roundings of its terms, the largest of which is scale |dg|
        # max (their sum under a softmax at most as large again), and of what is added
        size = 2 * abs(self.a["scale"]) * np.abs(n(self.dg)).max(1, keepdims=True) * self.k
        size = np.broadcast_to(size, l.shape) + (0.0 if self.extra is None else np.abs(n(self.extra)))
        ddl = 64 * U32 * size
        dl = np.abs(B.dlogits(l, idx, n(self.dg), *a)) + (0.0 if self.extra is None else np.abs(n(self.extra)))
        absx, absw = np.abs(n(self.x)), np.abs(n(self.w))
        own = 0.0
        if rep:
            own = np.zeros_like(dx)
            for t in range(self.T):
                for p in rep["slot_pos"][t]:
                    if p >= 0 and rep["rep_of_pos"][p] == p:
                        own[t] += np.abs(rep["dx_rep"][rep["rep_row"][p]])
        bound = ddl @ absw + 80 * U32 * (dl @ absw + own) + 1.01 * HALF[self.dtype] * np.abs(dx)
        assert (np.abs(numpy(out["dx"]) - dx) <= bound).all(), "dx"
        chain = (self.T + 80) * U32
        assert (np.abs(numpy(out["dw_gate"]) - dw) <= ddl.T @ absx + chain * (dl.T @ absx)).all(), "dw"
        assert (np.abs(numpy(out["db_gate"]) - db) <= ddl.sum(0) + chain * dl.sum(0)).all(), "db"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score,renorm", itertools.product(("softmax", "sigmoid"), (False, True)))
@pytest.mark.parametrize("T,d,E,k,extra,reps,capacity", [
    (1, 64, 4, 2, True, True, False), (130, 320, 13, 3, False, True, True), (333, 192, 64, 8, True, False, False),
    (70, 2112, 24, 6, False, True, False)])
def test_gradients(T, d, E, k, extra, reps, capacity, score, renorm, dtype):
    g = Gradients(T + E, dtype, T, d, E, k, score, renorm, extra, reps, capacity)
    g.check(g.run())


@pytest.mark.parametrize("dtype,T,d,E,k", [("bf16", 3001, 256, 64, 8), ("f32", 2500, 320, 8, 2),
                                            ("bf16", 2100, 1024, 16, 2)])
def test_gradients_of_many_tokens(dtype, T, d, E, k):
    g = Gradients(T, dtype, T, d, E, k, "sigmoid", True, False, True)
    out = g.run()
    g.check(out)
    again = g.run()
    assert all(g.torch.equal(out[n], again[n]) for n in ("dx", "dw_gate", "db_gate"))


def test_gradients_of_rows_past_4_gib():
    """bf16 rows of 9 GB: more parts than the chip alone asks for, each within 32-bit
    offsets.  All rows but a few are zero, at both ends and at every part's edges."""
    import torch
    import paper_2411_15419_amd as L
    T, d, E, k = 140000, 32768, 2, 1
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    some = sorted({t for p in range(1, 8) for at in (T * p // 8, T * p // 3, T * p // 4) for t in (at - 1, at, at + 63)
                   if 0 <= t < T} | {0, 1, T - 2, T - 1, 65535, 65536, 70015, 70016})
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    x[some] = torch.randn(len(some), d, generator=gen, device="cuda").bfloat16()
    w = torch.randn(E, d, generator=gen, device="cuda").bfloat16()
    l = torch.randn(T, E, generator=gen, device="cuda")
    idx, dg = l.argmax(1, keepdim=True).int(), torch.randn(T, k, generator=gen, device="cuda")
    dx, dw = torch.full_like(x, float("nan")), torch.empty(E, d, device="cuda")
    ws = torch.empty(L.route_scored_backward_workspace_size(T, d, E), dtype=torch.uint8, device="cuda")
    L.luffy_route_scored_backward(x, w, "sigmoid", l, idx, dg, dx, dw, None, ws, renormalise=False)
    s = torch.sigmoid(l.double().gather(1, idx.long()))
    dl = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, idx.long(), dg.double() * s * (1 - s))
    want, size = dl[some].t() @ x[some].double(), dl[some].t().abs() @ x[some].double().abs()
    # dl to 8 roundings, and a sum of `some` terms that are not zero, in at most 64 parts
    assert bool(((dw.double() - want).abs() <= (8 + len(some) + 64) * U32 * size).all())
    for t in (0, 65535, 65536, 131072, T - 1):     # offsets past 32 bits
        want = dl[t] @ w.double()
        assert bool(((dx[t].double() - want).abs() <= 1.01 * 2.0 ** -8 * want.abs()).all())
    assert not bool(torch.isnan(dx[::997]).any())


def test_gradients_of_extreme_logits():
    """Scores that under- and overflow float32 when taken by themselves."""
    for score in ("softmax", "sigmoid"):
        g = Gradients(5, "f32", 40, 64, 8, 3, score, True, False, False)
        g.l[:20] -= 150.0
        g.l[20:] *= 60.0
        g.idx = tensor(B.choose(numpy(g.l), 3, score), "i32")
        out = g.run()
        assert all(bool(g.torch.isfinite(out[n]).all()) for n in ("dx", "dw_gate", "db_gate"))
        if score == "softmax":
            g.check(out)
    r = Router(6, "f32", 30, 64, 8, 3, "sigmoid", False, renorm=True)
    r.b = r.b - 200.0
    r.check(r.run())


def test_indices_out_of_range_are_left_out():
    g = Gradients(7, "f32", 20, 64, 8, 2, "sigmoid", False, False, False)
    want = g.run()
    g.idx[3, 1], g.idx[4, 0] = -1, 8
    got = g.run()
    rows = [t for t in range(20) if t not in (3, 4)]
    assert g.torch.equal(want["dx"][rows], got["dx"][rows]) and bool(g.torch.isfinite(got["dx"]).all())


def test_gradients_captured():
    import torch
    g = Gradients(31, "bf16", 500, 256, 32, 4, "sigmoid", True, True, True)
    out = g.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.run(out)
    for scale in (1.0, -2.0, 0.5):
        g.dg.mul_(scale)
        graph.replay()
        want = g.run()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], out[n]) for n in ("dx", "dw_gate", "db_gate"))
