"""Norms with gate and residual on the GPU, forward and backward, against their
64-bit forms."""
import itertools

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24     # half a unit in the last place of float32, relative
HALF = {"f32": U32, "bf16": 2.0 ** -8}
# A row's sum adds at most 32 values a lane, then six lanes' and 16 waves' sums: 60
# roundings one after the other, each relative to the terms' absolute sum.  A
# result goes through two such sums (mean, variance) and a gradient through up to
# four (those of o and of y), with a dozen products between: 512 roundings of the
# sum of the terms' absolute values are more than can add up.
ROW = 512 * U32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def tensor(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()


def numpy(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, seed, dtype, T, d, norm, post, gate, pre, bias, eps=1e-5, alpha=0.8):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.T, self.d, self.norm, self.eps, self.alpha = dtype, T, d, norm, eps, alpha
        rows = lambda: rng.standard_normal((T, d)) * np.exp(0.5 * rng.standard_normal(d)) + 0.1  # noqa: E731
        self.t = {n: tensor(rows(), dtype) for n in ("x", "y", "o", "dout", "du")}
        vec = lambda at: tensor(at + 0.1 * rng.standard_normal(d), "f32")  # noqa: E731
        self.w = dict(w_post=vec(1.0) if post else None, b_post=vec(0.0) if post and bias else None,
                      w_pre=vec(1.0) if pre else None, b_pre=vec(0.0) if pre and bias else None,
                      gate={"none": None, "channel": vec(0.5), "token": tensor(rng.uniform(0, 1, (T, d)), dtype)}[gate])
        self.pre, self.torch = pre, torch
        self.n = {n: None if t is None else numpy(t) for n, t in {**self.t, **self.w}.items()}

    def empty(self, like):
        return None if like is None else self.torch.full_like(like, float("nan"))

    def forward(self):
        import paper_2411_15419_amd as L
        o, u = self.empty(self.t["x"]), self.empty(self.t["x"]) if self.pre else None
        L.luffy_block_norm(self.t["x"], self.t["y"], o, u, norm=self.norm, eps=self.eps, res_scale=self.alpha, **self.w)
        return o, u

    def backward(self, dout=True, du=True):
        import paper_2411_15419_amd as L
        t, w = self.t, self.w
        dx, dy = self.empty(t["x"]), self.empty(t["x"])
        du = du and self.pre
        got = dict(dgate=self.empty(w["gate"]), dw_post=self.empty(w["w_post"]),
                   db_post=self.empty(w["w_post"]), dw_pre=self.empty(w["w_pre"]) if du else None,
                   db_pre=self.empty(w["w_pre"]) if du else None)
        ws = self.torch.empty(L.block_norm_backward_workspace_size(self.T, self.d), dtype=self.torch.uint8, device="cuda")
        L.luffy_block_norm_backward(t["y"], t["o"], t["dout"] if dout else None, t["du"] if du else None, dx, dy, ws,
                                    norm=self.norm, eps=self.eps, res_scale=self.alpha, w_post=w["w_post"],
                                    b_post=w["b_post"], gate=w["gate"], w_pre=w["w_pre"] if du else None, **got)
        return dict(dx=dx, dy=dy, **{n: v for n, v in got.items() if v is not None})

    def reference(self, dout=True, du=True):
        n = self.n
        return B.block_norm_backward(n["y"], n["o"], n["dout"] if dout else None,
                                     n["du"] if du and self.pre else None, norm=self.norm, eps=self.eps,
                                     res_scale=self.alpha, w_post=n["w_post"], b_post=n["b_post"], gate=n["gate"],
                                     w_pre=n["w_pre"])

    def sizes(self, du=True):
        """The absolute sums that the gradients' terms can reach: the same formulas
        with every sign positive."""
        n = self.n
        mag = lambda a: 0.0 if a is None else np.abs(a)  # noqa: E731
        out = {}
        total = mag(n["dout"])

        def through(q, a):
            hat, r = B.norm_rows(a, self.norm, self.eps)
            hat = np.abs(hat) + r * np.abs(a).mean(1, keepdims=True)    # the deviation's own cancellation
            return r * (q + hat * (q * hat).mean(1, keepdims=True) + q.mean(1, keepdims=True)), hat

        if self.pre and du:
            g, ohat = through(mag(n["du"]) * mag(n["w_pre"]), n["o"])
            total = total + g
            out["dw_pre"], out["db_pre"] = (mag(n["du"]) * ohat).sum(0), mag(n["du"]).sum(0)
        out["dx"] = self.alpha * total
        v, dv = mag(n["y"]), total
        if n["w_post"] is not None:
            hat = through(0.0 * total, n["y"])[1]
            v = hat * mag(n["w_post"]) + mag(n["b_post"])
        if n["gate"] is not None:
            out["dgate"] = (total * v).sum(0) if n["gate"].ndim == 1 else total * v
            dv = total * mag(n["gate"])
        if n["w_post"] is not None:
            out["dw_post"], out["db_post"] = (dv * hat).sum(0), dv.sum(0)
            dv = through(dv * mag(n["w_post"]), n["y"])[0]
        out["dy"] = dv
        return out

    def check_forward(self, o, u):
        n = self.n
        kw = dict(norm=self.norm, eps=self.eps)

        def size(a, w, b):
            r = B.norm_rows(a, self.norm, self.eps)[1]
            return r * (np.abs(a) + np.abs(a).mean(1, keepdims=True)) * np.abs(w) + (0.0 if b is None else np.abs(b))

        ref = B.block_norm(n["x"], n["y"], res_scale=self.alpha, w_post=n["w_post"], b_post=n["b_post"], gate=n["gate"],
                           **kw)
        mag = np.abs(n["y"]) if n["w_post"] is None else size(n["y"], n["w_post"], n["b_post"])
        mag = self.alpha * np.abs(n["x"]) + mag * (1.0 if n["gate"] is None else np.abs(n["gate"]))
        o = numpy(o)
        assert (np.abs(o - ref) <= ROW * mag + HALF[self.dtype] * np.abs(ref) * 1.01).all(), "o"
        if u is not None:     # of o as it was stored
            ref = B.pre_norm(o, w_pre=n["w_pre"], b_pre=n["b_pre"], **kw)
            mag = size(o, n["w_pre"], n["b_pre"])
            assert (np.abs(numpy(u) - ref) <= ROW * mag + HALF[self.dtype] * np.abs(ref) * 1.01).all(), "u"

    def check_backward(self, got, dout=True, du=True):
        ref, size = self.reference(dout, du), self.sizes(du)
        # sums over rows: a chain of at most T more additions
        for name, t in got.items():
            half = HALF["f32" if t.dtype == self.torch.float32 else "bf16"]
            bound = (ROW + (self.T * U32 if t.dim() == 1 else 0.0)) * size[name] + half * np.abs(ref[name]) * 1.01
            bad = np.abs(numpy(t) - ref[name]) > bound
            assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist())


SHAPES = [(1, 64), (5, 192), (37, 512), (130, 576), (67, 1024), (33, 1088), (9, 2048), (6, 2112), (5, 4096), (3, 4160),
          (3, 8192), (2, 8256), (2, 16384), (3, 16448), (2, 32768)]
KINDS = list(itertools.product(("rms", "layer"), (False, True), ("none", "channel", "token"), (False, True)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_sizes(T, d, dtype):
    c = Case(T + d, dtype, T, d, "layer", True, "token", True, True)
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [320, 2240])
@pytest.mark.parametrize("norm,post,gate,pre", KINDS)
def test_parts(norm, post, gate, pre, d, dtype):
    c = Case(7, dtype, 43, d, norm, post, gate, pre, norm == "layer")
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("T,d", [(3001, 256), (1100, 1024), (700, 2560)])
def test_many_rows(T, d):
    """More rows than the grid has teams: every team takes several."""
    c = Case(11, "bf16", T, d, "rms", True, "channel", True, False)
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1536, 1600, 2560, 2624, 3008, 3136, 3584, 3648, 4608, 5120, 5184, 6144, 6208, 7232])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_teams_of_any_number_of_waves(norm, d, dtype):
    """Rows on three, five, six and seven waves, of all lanes or not, more of them than
    a block has teams."""
    c = Case(d, dtype, 7, d, norm, True, "channel", True, norm == "layer")
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


@pytest.mark.parametrize("T,d", [(1600, 1152), (1100, 2176), (1050, 2880)])
def test_more_rows_than_teams_of_odd_waves(T, d):
    c = Case(12, "bf16", T, d, "layer", True, "token", True, True)
    c.check_forward(*c.forward())
    c.check_backward(c.backward())


def test_more_rows_than_a_grid_has_blocks():
    """Past 2^20 rows a block takes several: rows at both ends and at the seam have the
    bits of a call of their own."""
    import torch
    import paper_2411_15419_amd as L
    T, d = (1 << 20) + 7, 576
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.randn(T, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
    o, u = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    kw = dict(norm="layer", res_scale=0.5, w_post=w, w_pre=w, gate=w)
    L.luffy_block_norm(x, y, o, u, **kw)
    some = [0, 1, 12345, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T - 1]
    o2, u2 = torch.empty(len(some), d, dtype=x.dtype, device="cuda"), torch.empty(len(some), d, dtype=x.dtype, device="cuda")
    L.luffy_block_norm(x[some], y[some], o2, u2, **kw)
    assert torch.equal(o[some], o2) and torch.equal(u[some], u2)
    assert not bool(torch.isnan(u).any())


def test_u_is_that_of_the_stored_stream():
    """u of a call with y and u of a call that is given o alone: the same bits."""
    import paper_2411_15419_amd as L
    c = Case(5, "bf16", 21, 1088, "layer", True, "channel", True, True)
    o, u = c.forward()
    again = c.empty(u)
    L.luffy_block_norm(o, None, None, again, norm="layer", eps=c.eps, w_pre=c.w["w_pre"], b_pre=c.w["b_pre"])
    assert c.torch.equal(u, again)


def test_first_norm_alone():
    """y None: u of the stream, and dx of its gradient and the stream's."""
    import torch
    import paper_2411_15419_amd as L
    c = Case(6, "f32", 19, 448, "layer", False, "none", True, True)
    t, n = c.t, c.n
    u, dx, dw = c.empty(t["x"]), c.empty(t["x"]), c.empty(c.w["w_pre"])
    L.luffy_block_norm(t["o"], None, None, u, norm="layer", eps=c.eps, w_pre=c.w["w_pre"], b_pre=c.w["b_pre"])
    ref = B.pre_norm(n["o"], norm="layer", eps=c.eps, w_pre=n["w_pre"], b_pre=n["b_pre"])
    assert np.abs(numpy(u) - ref).max() <= 1e-5 * np.abs(ref).max()
    ws = torch.empty(L.block_norm_backward_workspace_size(19, 448), dtype=torch.uint8, device="cuda")
    for dout in (None, t["dout"]):
        L.luffy_block_norm_backward(None, t["o"], dout, t["du"], dx, None, ws, norm="layer", eps=c.eps,
                                    w_pre=c.w["w_pre"], dw_pre=dw)
        ref = B.block_norm_backward(None, n["o"], None if dout is None else n["dout"], n["du"], norm="layer",
                                    eps=c.eps, w_pre=n["w_pre"])
        # 512 roundings of terms a few times the largest result
        assert np.abs(numpy(dx) - ref["dx"]).max() <= 4 * ROW * np.abs(ref["dx"]).max()
        assert np.abs(numpy(dw) - ref["dw_pre"]).max() <= 4 * ROW * np.abs(n["du"]).sum(0).max()


def test_without_the_next_norm():
    """du None: the stream's gradient alone; dout None is in test_first_norm_alone."""
    c = Case(8, "bf16", 29, 640, "rms", True, "token", True, False)
    c.check_backward(c.backward(du=False), du=False)


def test_rows_keep_to_themselves():
    """A row of NaN or infinities leaves the other rows as they were."""
    c = Case(9, "bf16", 24, 320, "layer", True, "channel", True, True)
    o, u = c.forward()
    c.t["y"][3, 5], c.t["x"][7, 0] = float("nan"), float("inf")
    o2, u2 = c.forward()
    keep = [r for r in range(24) if r not in (3, 7)]
    assert c.torch.equal(o[keep], o2[keep]) and c.torch.equal(u[keep], u2[keep])
    assert c.torch.isnan(u2[3]).all() and c.torch.isnan(u2[7]).any()


def test_large_mean_is_no_loss():
    """Deviations a thousand times smaller than the mean: sums of squares would lose
    them, sums of squared deviations do not."""
    c = Case(10, "f32", 16, 1024, "layer", True, "none", True, True)
    for name in ("y", "o"):
        c.t[name] += 1000.0
        c.n[name] = numpy(c.t[name])
    c.check_forward(*c.forward())
    c.check_backward(c.backward())
    o, _ = c.forward()
    ref = B.block_norm(c.n["x"], c.n["y"], res_scale=c.alpha, norm="layer", eps=c.eps, w_post=c.n["w_post"],
                       b_post=c.n["b_post"])
    # 64 roundings of the mean (1000 u each) over deviations of about one
    assert np.abs(numpy(o) - ref).max() <= 64 * 1000 * U32 * 4


def test_runs_repeat_bit_for_bit():
    c = Case(12, "bf16", 1500, 1024, "layer", True, "channel", True, True)
    a, b = c.backward(), c.backward()
    assert all(c.torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("T,d,norm,gate", [(8200, 2112, "layer", "channel"), (16401, 1088, "rms", "token"),
                                           (32771, 576, "layer", "token"), (4099, 4096, "rms", "channel"),
                                           (32775, 896, "rms", "token"), (32775, 896, "layer", "channel"),
                                           (16389, 1856, "layer", "token"), (8203, 3904, "layer", "channel"),
                                           (8203, 3904, "rms", "token"), (16399, 2048, "rms", "channel")])
def test_backward_of_many_rows(T, d, norm, gate):
    """bf16 rows in such numbers that the blocks hold two chunks a lane, where those fill
    the lanes; against the same formulas in float64 by autograd."""
    import torch
    import paper_2411_15419_amd as L
    gen = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    y, x, dout, du = (rnd(T, d).bfloat16() for _ in range(4))
    w = dict(w_post=1 + 0.1 * rnd(d), b_post=0.1 * rnd(d), w_pre=1 + 0.1 * rnd(d), b_pre=0.1 * rnd(d))
    gate = 0.5 + 0.1 * rnd(d) if gate == "channel" else (0.5 + 0.1 * rnd(T, d)).bfloat16()
    if norm == "rms":
        w["b_post"] = w["b_pre"] = None
    kw = dict(norm=norm, eps=1e-5, res_scale=0.7)
    o, u = torch.empty_like(x), torch.empty_like(x)
    L.luffy_block_norm(x, y, o, u, gate=gate, **w, **kw)

    def N(a, wt, b):
        c = a - a.mean(1, keepdim=True) if norm == "layer" else a
        return c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5) * wt + (0.0 if b is None else b)

    leaf = {n: t.double().requires_grad_() for n, t in dict(y=y, gate=gate, **w).items() if t is not None}
    x64 = x.double().requires_grad_()
    through = lambda n: leaf.get(n)  # noqa: E731
    o64 = 0.7 * x64 + leaf["gate"] * N(leaf["y"], leaf["w_post"], through("b_post"))
    stored = o64 + (o.double() - o64).detach()      # u is of o as it was stored
    ((stored * dout.double()).sum() + (N(stored, leaf["w_pre"], through("b_pre")) * du.double()).sum()).backward()
    got = dict(dx=torch.full_like(x, float("nan")), dy=torch.full_like(x, float("nan")),
               dgate=torch.full_like(gate, float("nan")),
               **{"d" + n: torch.full_like(t, float("nan")) for n, t in w.items() if t is not None})
    ws = torch.empty(L.block_norm_backward_workspace_size(T, d), dtype=torch.uint8, device="cuda")
    names = dict(w_post=w["w_post"], b_post=w["b_post"], gate=gate, w_pre=w["w_pre"])
    L.luffy_block_norm_backward(y, o, dout, du, workspace=ws, **names, **kw, **got)
    want = dict(dx=x64.grad, **{"d" + n: t.grad for n, t in leaf.items()})
    for n, t in got.items():
        # an entry is a sum of m terms, m the rows or one.  Over the entries, random as
        # they are, its root mean square is sqrt(m) of a term's; a term, a product of two
        # normal numbers, is below 32 of its own (5.6 sigma each), and m of them in
        # absolute value below 32 sqrt(m) root mean squares of the entries.
        m = T if t.dim() == 1 else 1
        half = HALF["f32"] if t.dtype == torch.float32 else HALF["bf16"]
        size = 32 * m ** 0.5 * want[n].square().mean().sqrt()
        bound = (ROW + (m - 1) * U32) * size + 1.01 * half * want[n].abs()
        assert bool(((t.double() - want[n]).abs() <= bound).all()), n
    again = {n: torch.empty_like(t) for n, t in got.items()}
    L.luffy_block_norm_backward(y, o, dout, du, workspace=ws, **names, **kw, **again)
    assert all(torch.equal(got[n], again[n]) for n in got)
