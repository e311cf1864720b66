"""Activations kept in microscaled 8 bits on the GPU: the format bit for bit, and
the experts' FFN forward and backward on them."""
import numpy as np
import pytest

from oracle import block_oracle as B
from oracle.luffy_oracle import activation, activation_grad

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
BF = 2.0 ** -8       # half a step of bf16, relative


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def tensor(a, dtype="bf16"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to({"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32}[dtype]).cuda()


def numpy(t):
    return t.double().cpu().numpy()


def awkward(rng, rows, cols):
    """Blocks of every kind: very different sizes, halfway cases, values that round
    to 128 steps, zeros, subnormals, the largest numbers, infinities and NaN."""
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, cols // 32)) * 5).repeat(32, 1)
    kinds = rng.integers(0, 12, (rows, cols // 32))
    for r in range(rows):
        for b in range(cols // 32):
            v = x[r, 32 * b:32 * b + 32]
            kind = kinds[r, b]
            if kind == 0:
                v[:] = 0.0
            elif kind == 1:
                v[:] = (rng.integers(-126, 126, 32) + 0.5) * 2.0 ** rng.integers(-20, 20)
                v[3] = 127.5 * 2.0 ** np.floor(np.log2(np.abs(v).max()) - 6)
            elif kind == 2:
                v[:] = rng.uniform(-1, 1, 32) * 127.99
                v[5], v[6] = 127.9, -127.9
            elif kind == 3:
                v[:] = rng.uniform(-1, 1, 32) * 1e-39
            elif kind == 4:
                v[:] = rng.uniform(-1, 1, 32) * 3.3e38
            elif kind == 5:
                v[rng.integers(0, 32)] = rng.choice([np.inf, -np.inf, np.nan])
            elif kind == 6:
                v[:] = 0.0
                v[7] = 2.0 ** -133
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (5, 1088), (130, 288), (67, 2048), (1, 11008), (2, 32768)])
def test_round_trip_bit_for_bit(rows, cols, dtype):
    import torch
    import paper_2411_15419_amd as L
    x = tensor(awkward(np.random.default_rng(rows + cols), rows, cols).astype(np.float32), dtype)
    q = torch.full((rows, cols), 99, dtype=torch.int8, device="cuda")
    s = torch.full(((cols + 255) // 256, rows, 8), 77, dtype=torch.uint8, device="cuda")
    L.luffy_mx8_quantize(x, q, s)
    ref_q, ref_s = B.mx8_quantize(numpy(x))
    assert np.array_equal(s.cpu().numpy(), B.pack_scales(ref_s))
    assert np.array_equal(q.cpu().numpy(), ref_q)
    for t in (torch.float32, torch.bfloat16):
        y = torch.full((rows, cols), 5.0, dtype=t, device="cuda")
        L.luffy_mx8_dequantize(q, s, y)
        assert np.array_equal(numpy(y), B.mx8_values(ref_q, ref_s), equal_nan=True)


def test_past_two_gigabytes():
    """Rows whose offsets leave 32 bits, in elements of the values and of the type."""
    import torch
    import paper_2411_15419_amd as L
    rows, cols = 70001, 32768
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    q = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    s = torch.empty(cols // 256, rows, 8, dtype=torch.uint8, device="cuda")
    L.luffy_mx8_quantize(x, q, s)
    y = torch.empty_like(x)
    L.luffy_mx8_dequantize(q, s, y)
    for r in (0, 32767, 65535, 65536, 65537, 70000):
        ref = B.mx8_rounded(numpy(x[r:r + 1]))
        assert np.array_equal(numpy(y[r:r + 1]), ref), r


class Ffn:
    def __init__(self, seed, counts, d, d_ff, act, index=True, dw="bf16"):
        import torch
        rng = np.random.default_rng(seed)
        E, R = len(counts), int(sum(counts))
        self.E, self.R, self.d, self.d_ff, self.act, self.torch, self.dw = E, R, d, d_ff, act, torch, dw
        self.max_rows = R + 5
        rows = R + 9 if index else self.max_rows
        self.x = tensor(rng.standard_normal((rows, d)) * np.exp(0.5 * rng.standard_normal(d)))
        self.index = None
        if index:
            self.index = tensor(np.concatenate([rng.integers(0, rows, R), np.full(5, 10 ** 9)]), "i32")
        self.off = tensor(np.concatenate([[0], np.cumsum(counts)]), "i32")
        self.w1 = tensor(rng.standard_normal((E, d_ff, d)) / np.sqrt(d))
        self.w2 = tensor(rng.standard_normal((E, d, d_ff)) / np.sqrt(d_ff))
        self.dy = tensor(rng.standard_normal((self.max_rows, d)))

    def forward(self):
        import paper_2411_15419_amd as L
        t = self.torch
        out = dict(zq=t.full((self.max_rows, self.d_ff), 99, dtype=t.int8, device="cuda"),
                   zs=t.full(((self.d_ff + 255) // 256, self.max_rows, 8), 77, dtype=t.uint8, device="cuda"),
                   y_rep=t.full((self.max_rows, self.d), -3.0, dtype=t.bfloat16, device="cuda"))
        ws = t.empty(L.expert_ffn_workspace_size(self.max_rows, self.E, self.d_ff, L.LUFFY_BF16), dtype=t.uint8,
                     device="cuda")
        L.luffy_expert_ffn_keep(self.x, self.index, self.off, self.w1, self.w2, self.act, self.max_rows,
                                workspace=ws, **out)
        return out

    def backward(self, f, x8=None):
        import paper_2411_15419_amd as L
        t = self.torch
        dw = t.bfloat16 if self.dw == "bf16" else t.float32
        out = dict(dx_rep=t.full((self.max_rows, self.d), -3.0, dtype=t.bfloat16, device="cuda"),
                   dw1=t.full(self.w1.shape, -3.0, dtype=dw, device="cuda"),
                   dw2=t.full(self.w2.shape, -3.0, dtype=dw, device="cuda"))
        ws = t.empty(L.expert_ffn_backward_kept_workspace_size(self.max_rows, self.E, self.d, self.d_ff),
                     dtype=t.uint8, device="cuda")
        x, xs = x8 if x8 else (self.x, None)
        L.luffy_expert_ffn_backward_kept(x, xs, self.index, self.off, self.w1, self.w2, self.act, self.max_rows,
                                         f["zq"], f["zs"], self.dy, workspace=ws, **out)
        return out

    def quantised_x(self):
        import paper_2411_15419_amd as L
        t = self.torch
        q = t.empty(self.x.shape, dtype=t.int8, device="cuda")
        s = t.empty(((self.d + 255) // 256, self.x.shape[0], 8), dtype=t.uint8, device="cuda")
        L.luffy_mx8_quantize(self.x, q, s)
        return q, s

    def rows(self, x):
        return x[self.index.cpu().numpy()[:self.R]] if self.index is not None else x[:self.R]

    def kept(self, f):
        s = B.unpack_scales(f["zs"].cpu().numpy(), self.d_ff)[:self.R]
        return B.mx8_values(f["zq"].cpu().numpy()[:self.R], s), np.ldexp(1.0, s.astype(int) - 127).repeat(32, 1)

    def by_expert(self):
        off = self.off.cpu().numpy()
        return [(e, slice(int(off[e]), int(off[e + 1]))) for e in range(self.E)]

    def check_forward(self, f):
        import paper_2411_15419_amd as L
        t = self.torch
        # y_rep: the bits of the FFN that keeps nothing
        y = t.full_like(f["y_rep"], -3.0)
        ws = t.empty(L.expert_ffn_workspace_size(self.max_rows, self.E, self.d_ff, L.LUFFY_BF16), dtype=t.uint8,
                     device="cuda")
        L.luffy_expert_ffn(self.x, self.index, self.off, self.w1, self.w2, self.act, self.max_rows, y, ws)
        assert t.equal(y, f["y_rep"])
        z, step = self.kept(f)
        x, w1 = self.rows(numpy(self.x)), numpy(self.w1)
        for e, r in self.by_expert():
            ref = x[r] @ w1[e].T
            err = (self.d / 16 + 64) * U32 * (np.abs(x[r]) @ np.abs(w1[e]).T)    # sums of 16 products and more a rounding
            edge = np.where(np.abs(ref) + err > 127.5 * step[r], 1.0, 0.5)
            assert (np.abs(z[r] - ref) <= edge * step[r] + err).all()
            most = np.abs(ref).reshape(ref.shape[0], self.d_ff // 32, 32).max(-1).repeat(32, 1)
            assert ((most <= 128 * step[r] + err) & (most >= 64 * step[r] - err)).all()
        assert bool((f["zq"][self.R:] == 99).all()) and bool((f["y_rep"][self.R:] == -3.0).all())
        s = f["zs"].cpu().numpy()
        assert (s[:, self.R:] == 77).all()
        used = self.d_ff // 32 - 8 * (s.shape[0] - 1)
        assert (s[-1, :self.R, used:] == 0).all()

    def check_backward(self, f, g, x):
        """x: the rows that dW1 takes, as values."""
        z, _ = self.kept(f)
        x, dy, w1, w2 = self.rows(x), numpy(self.dy)[:self.R], numpy(self.w1), numpy(self.w2)
        dx, dw1, dw2 = B.ffn_backward_kept(x, z, self.off.cpu().numpy(), w1, w2, self.act, dy)
        half = BF if self.dw == "bf16" else U32
        got = {n: numpy(v) for n, v in g.items()}
        for e, r in self.by_expert():
            n = r.stop - r.start
            slope, a = activation_grad(z[r], self.act), activation(z[r], self.act)
            # dz: the product's float32 sum, the slope's approximation (2^-20 of its
            # terms, which stay below 1.2), and bf16's rounding
            dz = np.abs(dy[r] @ w2[e]) * np.abs(slope)
            sums = (self.d / 16 + 64) * U32 * (np.abs(dy[r]) @ np.abs(w2[e]))
            ddz = sums * np.abs(slope) + 2.0 ** -20 * 2 * (np.abs(dy[r] @ w2[e]) + sums) + 1.01 * BF * dz
            # a: the approximation (2^-20 |z|) and the rounding
            da = 2.0 ** -20 * np.abs(z[r]) + 1.01 * BF * np.abs(a)
            tail = lambda k: (k / 16 + 64) * U32  # noqa: E731
            b = ddz @ np.abs(w1[e]) + tail(self.d_ff) * ((dz + ddz) @ np.abs(w1[e])) + 1.01 * BF * np.abs(dx[r])
            assert (np.abs(got["dx_rep"][r] - dx[r]) <= b).all(), ("dx", e)
            b = ddz.T @ np.abs(x[r]) + tail(n) * ((dz + ddz).T @ np.abs(x[r])) + 1.01 * half * np.abs(dw1[e])
            assert (np.abs(got["dw1"][e] - dw1[e]) <= b).all(), ("dw1", e)
            b = np.abs(dy[r]).T @ da + tail(n) * (np.abs(dy[r]).T @ (np.abs(a) + da)) + 1.01 * half * np.abs(dw2[e])
            assert (np.abs(got["dw2"][e] - dw2[e]) <= b).all(), ("dw2", e)
        assert (got["dx_rep"][self.R:] == -3.0).all()


SHAPES = [([1], 64, 64), ([3, 0, 5], 64, 320), ([37, 130, 1, 0], 192, 576), ([300, 20], 320, 256), ([257, 129], 128, 832),
          ([0, 0, 7], 512, 64)]


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("counts,d,d_ff", SHAPES)
def test_ffn_keep(counts, d, d_ff, act):
    c = Ffn(d + d_ff, counts, d, d_ff, act, dw="f32" if d == 192 else "bf16")
    f = c.forward()
    c.check_forward(f)
    c.check_backward(f, c.backward(f), numpy(c.x))
    x8 = c.quantised_x()
    c.check_backward(f, c.backward(f, x8), B.mx8_rounded(numpy(c.x)))


def test_ffn_keep_without_index():
    c = Ffn(3, [40, 9], 128, 192, "gelu", index=False, dw="f32")
    f = c.forward()
    c.check_forward(f)
    c.check_backward(f, c.backward(f), numpy(c.x))
    c.check_backward(f, c.backward(f, c.quantised_x()), B.mx8_rounded(numpy(c.x)))


def test_no_rows():
    c = Ffn(4, [0, 0], 64, 128, "silu")
    f = c.forward()
    g = c.backward(f)
    assert bool((f["zq"] == 99).all()) and bool((g["dx_rep"] == -3.0).all())
    assert not bool(g["dw1"].any()) and not bool(g["dw2"].any())


def test_rows_that_are_no_numbers_keep_to_themselves():
    c = Ffn(5, [33, 20], 128, 320, "gelu")
    clean = c.backward(c.forward())
    t = int(c.index[3])
    c.x[t, 5] = float("inf")
    f = c.forward()
    g = c.backward(f)
    same = [r for r in range(c.R) if int(c.index[r]) != t]
    assert bool((f["zs"][:, 3].flatten()[: 10] == 255).all())
    assert c.torch.equal(clean["dx_rep"][same], g["dx_rep"][same])
    assert bool(c.torch.isnan(g["dx_rep"][3]).all())


def test_repeat_capture_and_streams():
    import torch
    c = Ffn(6, [200, 90, 0, 310], 256, 512, "silu")
    f = c.forward()
    g = c.backward(f)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        f2 = c.forward()
        g2 = c.backward(f2)
    torch.cuda.synchronize()
    assert all(torch.equal(f[n], f2[n]) for n in f) and all(torch.equal(g[n], g2[n]) for n in g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f3 = c.forward()
        g3 = c.backward(f3)
    for k in range(3):
        c.x.copy_(tensor(np.random.default_rng(k).standard_normal(c.x.shape)))
        graph.replay()
        f = c.forward()
        g = c.backward(f)
        torch.cuda.synchronize()
        assert all(torch.equal(f[n], f3[n]) for n in f) and all(torch.equal(g[n], g3[n]) for n in g)
