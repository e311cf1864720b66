"""Microscaled 4-bit matrices on the GPU against their 64-bit forms:
quantisation and back (bit for bit), the product, the experts' FFN."""
import numpy as np
import pytest

from oracle import mx4_oracle as M

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24     # half a unit in the last place of float32, relative


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


def gpu(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def bf16(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).double().numpy()


def within(got, ref, bound, out):
    """Where got is what a value within bound of ref rounds to in its type
    (rounding keeps order, so the two ends are enough)."""
    import torch
    t = torch.float32 if out == "f32" else torch.bfloat16
    low, high = (torch.from_numpy(v).to(t).double().numpy() for v in (ref - bound, ref + bound))
    return (got >= low) & (got <= high)


def awkward_rows(rng, rows, cols):
    """Rows of every kind of block: normal, of very different sizes, halfway
    cases, zeros, subnormals, the largest numbers, infinities and NaN."""
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, cols // 32)) * 4).repeat(32, 1)
    kinds = rng.integers(0, 12, (rows, cols // 32))
    for r in range(rows):
        for b in range(cols // 32):
            v = x[r, 32 * b:32 * b + 32]
            kind = kinds[r, b]
            if kind == 0:
                v[:] = 0.0
            elif kind == 1:      # halfway cases under a scale of a power of two
                half = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0])
                v[:] = np.tile(half, 4) * rng.choice([-1, 1], 32) * 2.0 ** rng.integers(-20, 20)
            elif kind == 2:      # one value above the largest multiple
                v[:] = rng.uniform(-7.99, 7.99, 32)
                v[5] = 7.99
            elif kind == 3:
                v[:] = rng.uniform(-1, 1, 32) * 1e-39
            elif kind == 4:
                v[:] = rng.uniform(-3, 3, 32) * 1e38
            elif kind == 5:
                v[:] = 0.0
                v[rng.integers(32)] = 1e-30
            elif kind == 6 and r % 3 == 0:
                v[rng.integers(32)] = rng.choice([np.inf, -np.inf, np.nan])
    return x


def stored(x):
    q, s = M.pack(*M.quantize(x))
    return q, s


def launch_quantize(x, groups=1, row_index=None, rows=None):
    """x: torch [groups*rows, cols]; returns (values, scales) as numpy."""
    import torch
    import paper_2411_15419_amd as L
    n = (rows if rows is not None else x.shape[0] // groups)
    cols = x.shape[1]
    lead = (groups,) if groups > 1 else ()
    q = torch.full(lead + (n, cols // 2), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full(lead + ((cols + 255) // 256, n, 8), 0xA5, dtype=torch.uint8, device="cuda")
    L.luffy_mx4_quantize(x.view(lead + (n, cols)) if row_index is None else x, q, s, row_index=row_index)
    torch.cuda.synchronize()
    assert s.numel() == L.mx4_scale_bytes(groups, n, cols)
    return q.cpu().numpy(), s.cpu().numpy()


def same_values(q, s, code, scale):
    """Stored (q, s) holds exactly these codes (a zero's sign aside) and scales,
    and zeros past the last column."""
    rows, cols = code.shape
    got = np.empty((rows, cols), np.uint8)
    got[:, 0::2], got[:, 1::2] = q & 15, q >> 4
    flat = s.transpose(1, 0, 2).reshape(rows, -1)
    assert np.array_equal(flat[:, :cols // 32], scale)
    assert not flat[:, cols // 32:].any()
    finite = np.repeat(scale != 255, 32, axis=1)
    differ = (got != code) & ~(((got & 7) == 0) & ((code & 7) == 0)) & finite
    assert not differ.any(), np.argwhere(differ)[:5]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 64), (3, 96), (7, 256), (2, 288), (33, 1088), (130, 4096),
                                       (4097, 32)])
def test_quantize_matches_the_definition(rows, cols, dtype):
    import torch
    rng = np.random.default_rng(rows * 10007 + cols)
    x = torch.from_numpy(awkward_rows(rng, rows, cols).astype(np.float32))
    if dtype == "bf16":
        x = x.to(torch.bfloat16)
    code, scale = M.quantize(x.double().numpy())
    q, s = launch_quantize(x.cuda())
    same_values(q, s, code, scale)


def test_quantize_groups_and_row_index():
    import torch
    rng = np.random.default_rng(5)
    x = torch.from_numpy(awkward_rows(rng, 3 * 37, 320).astype(np.float32)).to(torch.bfloat16)
    q, s = launch_quantize(x.cuda(), groups=3)
    for g in range(3):
        same_values(q[g], s[g], *M.quantize(x[37 * g:37 * g + 37].double().numpy()))
    idx = rng.integers(0, 111, 50).astype(np.int32)
    q, s = launch_quantize(x.cuda(), row_index=gpu(idx), rows=50)
    same_values(q, s, *M.quantize(x.double().numpy()[idx]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dequantize_every_code_and_scale(dtype):
    """All 16 codes under all 256 scale bytes: exact in both types (a bf16
    holds two significant bits at every exponent used)."""
    import torch
    import paper_2411_15419_amd as L
    scale = np.arange(256, dtype=np.uint8)[:, None]
    code = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    q, s = M.pack(code, scale)
    out = torch.empty(256, 32, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    L.luffy_mx4_dequantize(gpu(q), gpu(s), out)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(M.values(code, scale)).to(out.dtype).double().numpy()
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[:255], want[:255])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups,rows,cols", [(1, 1, 32), (1, 77, 1088), (4, 19, 288)])
def test_round_trip(groups, rows, cols, dtype):
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(cols)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.from_numpy(rng.standard_normal((groups, rows, cols)).astype(np.float32)).to(t)
    q = torch.empty(groups, rows, cols // 2, dtype=torch.uint8, device="cuda")
    s = torch.empty(groups, (cols + 255) // 256, rows, 8, dtype=torch.uint8, device="cuda")
    y = torch.empty(groups, rows, cols, dtype=t, device="cuda")
    L.luffy_mx4_quantize(x.cuda(), q, s)
    L.luffy_mx4_dequantize(q, s, y)
    want = M.rounded(x.double().numpy().reshape(-1, cols)).reshape(groups, rows, cols)
    assert np.array_equal(y.double().cpu().numpy(), want)


def matmul_case(rng, n, E, N, K, out, spread=1.0, tail_rows=0):
    """Rows of the experts with n[e] rows each; returns got, reference, bound."""
    import torch
    import paper_2411_15419_amd as L
    R = int(sum(n))
    rows = max(1, R + tail_rows)
    x = M.quantize(rng.standard_normal((rows, K)) * np.exp(spread * rng.standard_normal((rows, 1))))
    w = [M.quantize(rng.standard_normal((N, K))) for _ in range(E)]
    wq, ws = zip(*[M.pack(*m) for m in w])
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    y = torch.full((rows, N), 768.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    xq, xs = M.pack(*x)
    L.luffy_mx4_matmul(gpu(xq), gpu(xs), gpu(off) if E > 1 or tail_rows else None, gpu(np.stack(wq)),
                       gpu(np.stack(ws)), y)
    got = y.double().cpu().numpy()
    xv = M.values(*x)
    ref, mag = np.zeros((R, N)), np.zeros((R, N))
    for e in range(E):
        wv = M.values(*w[e])
        sl = slice(off[e], off[e + 1])
        ref[sl], mag[sl] = xv[sl] @ wv.T, np.abs(xv[sl]) @ np.abs(wv.T)
    bound = K * U32 * mag     # K exact products, K - 1 additions in float32 in any order
    assert (got[R:] == 768.0).all() or tail_rows == 0, "rows past the last expert's were written"
    return got[:R], ref, bound


@pytest.mark.parametrize("m,N,K,out", [
    (1, 32, 32, "f32"), (1, 64, 64, "bf16"), (5, 96, 288, "f32"), (127, 128, 256, "bf16"), (128, 160, 512, "f32"),
    (129, 256, 1088, "bf16"), (300, 288, 96, "f32"), (64, 1120, 2016, "bf16"), (257, 544, 4096, "f32"),
    (17, 2880, 1088, "bf16"), (520, 320, 768, "bf16"), (33, 32, 8192, "f32")])
def test_matmul_one_expert(m, N, K, out):
    got, ref, bound = matmul_case(np.random.default_rng(m + N + K), [m], 1, N, K, out)
    assert within(got, ref, bound, out).all(), np.abs(got - ref).max()


@pytest.mark.parametrize("n,N,K,out", [
    ([0, 1, 0, 200, 33], 96, 320, "f32"), ([5], 64, 64, "f32"), ([0, 0, 0], 64, 64, "bf16"),
    ([130, 0, 260, 7, 1, 128], 288, 544, "bf16"), ([1] * 64, 64, 256, "f32"), ([3, 0] * 32, 128, 96, "bf16"),
    ([600, 2, 70], 320, 288, "f32")])
def test_matmul_by_expert(n, N, K, out):
    """Experts without rows, more rows than one tile, rows past the last expert
    that must stay as they are."""
    got, ref, bound = matmul_case(np.random.default_rng(len(n) * N + K), n, len(n), N, K, out, tail_rows=9)
    assert within(got, ref, bound, out).all(), np.abs(got - ref).max()


def test_matmul_not_a_number_stays_in_its_row_and_column():
    """A block without numbers makes its row of the result NaN (rows) or its
    column (weights), and nothing else."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(3)
    M_, N, K = 70, 96, 288
    x, w = rng.standard_normal((M_, K)), rng.standard_normal((N, K))
    x[11, 40] = np.nan
    x[69, 280] = np.inf
    w[33, 5] = -np.inf
    xv, wv = M.quantize(x), M.quantize(w)
    y = torch.empty(M_, N, device="cuda")
    (xq, xs), (wq, ws) = M.pack(*xv), M.pack(*wv)
    L.luffy_mx4_matmul(gpu(xq), gpu(xs), None, gpu(wq[None]), gpu(ws[None]), y)
    got = y.double().cpu().numpy()
    want = np.zeros((M_, N), bool)
    want[[11, 69]] = True
    want[:, 33] = True
    assert np.array_equal(np.isnan(got), want)
    a, b = np.nan_to_num(M.values(*xv)), np.nan_to_num(M.values(*wv))
    ok = ~want
    assert (np.abs(got - a @ b.T)[ok] <= (K * U32 * (np.abs(a) @ np.abs(b.T)))[ok]).all()


def ffn_reference(x, off, w1, w2, act):
    """64-bit result, and a bound on what float32 sums may change: a hidden value
    within the float32 error of a halfway point (or whose block's largest value
    is within it of a power of two) may be rounded to the neighbour."""
    R, E = x.shape[0], len(w1)
    d, d_ff = w2[0].shape
    y, bound = np.zeros((R, d)), np.zeros((R, d))
    xv = M.rounded(x)
    for e in range(E):
        sl = slice(off[e], off[e + 1])
        if off[e + 1] == off[e]:
            continue
        z = xv[sl] @ w1[e].T
        ez = xv.shape[1] * U32 * (np.abs(xv[sl]) @ np.abs(w1[e].T))
        h = M.activation(z, act)
        eh = 1.13 * ez + 8 * U32 * np.abs(z) + 8 * U32 * np.abs(h)     # |act'| <= 1.13; erff, expf within a few ulp
        hv = M.rounded(h)
        off_by = np.maximum(np.abs(M.rounded(h - eh) - hv), np.abs(M.rounded(h + eh) - hv))
        # a block whose scale may change: every value by up to a step of the coarser one
        blk = np.abs(h).reshape(h.shape[0], -1, 32)
        eb = eh.reshape(blk.shape).max(-1)
        top = blk.max(-1)
        flips = np.floor(np.log2(np.maximum(top - eb, 1e-300))) != np.floor(np.log2(top + eb))
        step = np.where(flips, top, 0.0)
        off_by = np.maximum(off_by, np.repeat(step, 32, axis=1))
        y[sl] = hv @ w2[e].T
        mag = np.abs(hv) @ np.abs(w2[e].T)
        bound[sl] = off_by @ np.abs(w2[e].T) + d_ff * U32 * mag
    return y, bound


@pytest.mark.parametrize("n,d,d_ff,act", [
    ([1], 64, 64, "gelu"), ([0, 3, 0, 40], 128, 320, "silu"), ([129, 0, 31, 260], 192, 576, "gelu"),
    ([2] * 32, 256, 256, "silu"), ([70, 200], 1088, 832, "gelu")])
def test_expert_ffn(n, d, d_ff, act):
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(d + d_ff)
    E, R = len(n), int(sum(n))
    tokens = R + 5
    x = bf16(rng.standard_normal((tokens, d)) * np.exp(0.5 * rng.standard_normal(d)))
    index = rng.integers(0, tokens, R + 7).astype(np.int32)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    w1 = [M.quantize(0.05 * rng.standard_normal((d_ff, d))) for _ in range(E)]
    w2 = [M.quantize(0.05 * rng.standard_normal((d, d_ff))) for _ in range(E)]
    q1, s1 = map(np.stack, zip(*[M.pack(*m) for m in w1]))
    q2, s2 = map(np.stack, zip(*[M.pack(*m) for m in w2]))
    max_rows = R + 7                          # an upper bound, as T * k is
    xt = gpu(x.astype(np.float32), torch.bfloat16)
    y = torch.full((max_rows, d), 768.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.mx4_expert_ffn_workspace_size(max_rows, E, d, d_ff),), 0xFF, dtype=torch.uint8, device="cuda")
    args = (gpu(off), gpu(q1), gpu(s1), gpu(q2), gpu(s2), act, max_rows)
    L.luffy_mx4_expert_ffn(xt, gpu(index), *args, y, ws)
    got = y.double().cpu().numpy()
    assert (got[R:] == 768.0).all()
    ref, bound = ffn_reference(x[index[:R]], off, [M.values(*m) for m in w1], [M.values(*m) for m in w2], act)
    bad = ~within(got[:R], ref, bound, "bf16")
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got[:R] - ref).max())
    # rows read in place give the same, and so does a second call on the used workspace
    z = torch.full((max_rows, d), 768.0, dtype=torch.bfloat16, device="cuda")
    L.luffy_mx4_expert_ffn(xt[gpu(index).long()].contiguous(), None, *args, z, ws)
    assert torch.equal(y, z)


def test_calls_replay_in_a_graph_and_run_on_another_stream():
    """Captured once, replayed on new inputs with eager work between: the
    same as the eager calls, bit for bit; and the calls on a side stream."""
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(9)
    E, d, d_ff, R = 3, 256, 320, 90
    off = gpu(np.array([0, 40, 40, 90], np.int32))
    w = [[M.pack(*M.quantize(0.05 * rng.standard_normal(s))) for _ in range(E)] for s in ((d_ff, d), (d, d_ff))]
    q1, s1 = (gpu(np.stack(a)) for a in zip(*w[0]))
    q2, s2 = (gpu(np.stack(a)) for a in zip(*w[1]))
    x = torch.empty(R, d, dtype=torch.bfloat16, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(L.mx4_expert_ffn_workspace_size(R, E, d, d_ff), dtype=torch.uint8, device="cuda")

    def call(out, stream=None):
        L.luffy_mx4_expert_ffn(x, None, off, q1, s1, q2, s2, "gelu", R, out, ws, stream=stream)

    x.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(y)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
    for _ in range(4):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        call(z, side)
        side.synchronize()
        assert torch.equal(y, z)
