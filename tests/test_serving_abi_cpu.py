"""The serving entry points refuse bad arguments on the host, before anything
is enqueued, and size their buffers (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2411_15419_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2411_15419_amd import build
        build.build()
    return L.load_library()


FAKE = ctypes.c_void_p(256)     # never dereferenced: the checks fail first
ODD = ctypes.c_void_p(264)      # 8-byte aligned only
BYTE = ctypes.c_void_p(257)


def caller(fn, good):
    def call(**change):
        a = list(good)
        for i, v in change.items():
            a[int(i[1:])] = v
        return fn(*a)
    return call


def test_scale_bytes(lib):
    assert lib.luffy_mx4_scale_bytes(1, 1, 32) == 8
    assert lib.luffy_mx4_scale_bytes(3, 5, 256) == 3 * 5 * 8
    assert lib.luffy_mx4_scale_bytes(3, 5, 288) == 3 * 5 * 16
    assert lib.luffy_mx4_scale_bytes(64, 32768, 32768) == 64 * 32768 * 128 * 8
    assert lib.luffy_mx4_scale_bytes(0, 5, 288) == 0


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
def test_quantize_refusals(lib, name):
    if name == "quantize":
        call = caller(lib.luffy_mx4_quantize, [FAKE, None, 1, 4, 64, 0, FAKE, FAKE, None])
        x, g, r, c, t, q, s = "a0 a2 a3 a4 a5 a6 a7".split()
        assert call(a1=FAKE, a2=2) == -1                 # row_index with several groups
    else:
        call = caller(lib.luffy_mx4_dequantize, [FAKE, FAKE, 1, 4, 64, 0, FAKE, None])
        q, s, g, r, c, t, x = "a0 a1 a2 a3 a4 a5 a6".split()
    for ptr in (x, q, s):
        assert call(**{ptr: None}) == -1
    for size in (g, r, c):
        assert call(**{size: 0}) == -1 and call(**{size: -3}) == -1
    assert call(**{t: 2}) == -1                          # 4-bit is no input type
    assert call(**{c: 48}) == -2                         # no whole blocks
    assert call(**{x: ODD}) == -1 and call(**{q: ODD}) == -1 and call(**{s: BYTE}) == -1
    assert call(**{g: 64, r: 2 ** 31 - 1, c: 32768}) == -2


def test_matmul_refusals(lib):
    call = caller(lib.luffy_mx4_matmul, [FAKE, FAKE, 4, FAKE, 2, 64, 64, FAKE, FAKE, FAKE, 0, None])
    for p in (0, 1, 7, 8, 9):
        assert call(**{f"a{p}": None}) == -1
    assert call(a3=None) == -1                           # two experts without offsets
    for p in (2, 4, 5, 6):
        assert call(**{f"a{p}": 0}) == -1
    assert call(a10=2) == -1
    assert call(a4=65) == -2
    assert call(a5=48) == -2 and call(a6=40) == -2 and call(a5=32800) == -2 and call(a6=32800) == -2
    assert call(a2=(1 << 24) + 1) == -2
    for p in (0, 7, 9):
        assert call(**{f"a{p}": ODD}) == -1
    for p in (1, 8):
        assert call(**{f"a{p}": BYTE}) == -1


def test_expert_ffn_refusals(lib):
    need = lib.luffy_mx4_expert_ffn_workspace_size(8, 2, 64, 128)
    assert need > 0 and lib.luffy_mx4_expert_ffn_workspace_size(0, 2, 64, 128) == 0
    call = caller(lib.luffy_mx4_expert_ffn, [FAKE, None, FAKE, 2, 64, 128, FAKE, FAKE, FAKE, FAKE, 0, 8, FAKE, FAKE,
                                             need - 1, None])
    for p in (0, 2, 6, 7, 8, 9, 12):
        assert call(**{f"a{p}": None}) == -1
    for p in (3, 4, 5, 11):
        assert call(**{f"a{p}": 0}) == -1
    assert call(a10=2) == -1
    assert call(a3=65) == -2 and call(a4=96) == -2 and call(a5=32) == -2 and call(a11=(1 << 24) + 1) == -2
    for p in (0, 6, 8, 12):
        assert call(**{f"a{p}": ODD}) == -1
    for p in (7, 9):
        assert call(**{f"a{p}": BYTE}) == -1
    assert call() == -3                                   # one byte short
    assert call(a14=1 << 30, a13=None) == -3 and call(a14=1 << 30, a13=ODD) == -3
    assert b"workspace" in lib.luffy_last_error()


def test_moe_few_refusals(lib):
    need = lib.luffy_moe_few_workspace_size(4, 64, 4, 2, 128)
    assert need > 0
    assert lib.luffy_moe_few_workspace_size(65, 64, 4, 2, 128) == 0
    assert lib.luffy_moe_few_workspace_size(4, 64, 4, 3, 128) == 0
    good = [FAKE, 4, 64, 1, FAKE, None, 4, 2, FAKE, None, FAKE, None, 1, 128, 0, FAKE, FAKE, FAKE, FAKE, need - 1, None]
    call = caller(lib.luffy_moe_few, good)
    for p in (0, 4, 8, 10, 15, 16, 17):
        assert call(**{f"a{p}": None}) == -1
    for p in (1, 2, 6, 13):
        assert call(**{f"a{p}": 0}) == -1
    assert call(a7=3) == -1 and call(a6=1, a7=2) == -1    # k
    assert call(a3=2) == -1 and call(a12=0) == -1 and call(a12=3) == -1 and call(a14=2) == -1
    assert call(a12=2) == -1                              # 4-bit weights without scales
    assert call(a12=2, a9=FAKE) == -1
    assert call(a3=0, a12=2, a9=FAKE, a11=FAKE) == -2     # 4-bit weights under float32
    assert call(a1=65) == -2 and call(a6=65) == -2 and call(a2=96) == -2 and call(a13=32832) == -2
    for p in (0, 4, 8, 10):
        assert call(**{f"a{p}": ODD}) == -1
    assert call() == -3 and call(a19=1 << 30, a18=ODD) == -3


def test_binding_refusals(lib):
    """Shapes and types that the binding can tell from the tensors."""
    import torch
    import paper_2411_15419_amd as L
    u8 = dict(dtype=torch.uint8)
    q, s = torch.zeros(4, 32, **u8), torch.zeros(1, 4, 8, **u8)
    with pytest.raises(L.LuffyError, match="GPU"):
        L.luffy_mx4_quantize(torch.zeros(4, 64), q, s)
    with pytest.raises(L.LuffyError, match="scales"):
        L.luffy_mx4_quantize(torch.zeros(4, 64), q, torch.zeros(4, 8, **u8))
    with pytest.raises(L.LuffyError, match="fit"):
        L.luffy_mx4_quantize(torch.zeros(5, 64), q, s)
    with pytest.raises(L.LuffyError, match="uint8"):
        L.luffy_mx4_dequantize(q.int(), s, torch.zeros(4, 64))
    with pytest.raises(L.LuffyError, match="rows"):
        L.luffy_mx4_matmul(q, s, None, q[None], s[None], torch.zeros(4, 5))
    with pytest.raises(L.LuffyError, match="both scales"):
        L.luffy_moe_few(torch.zeros(1, 64), torch.zeros(4, 64), None, q[None], q[None], 1, "gelu", None, None, None,
                        None, w1_scale=s[None])
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    w = torch.zeros(4, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(L.LuffyError, match="w_gate"):
        L.luffy_moe_few(x, torch.zeros(4, 128), None, w, w, 1, "gelu", None, None, x, None)
    with pytest.raises(L.LuffyError, match="b_gate"):
        L.luffy_moe_few(x, torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(3), w, w, 1, "gelu", None, None, x,
                        None)


def test_reference_rounding_is_nearest_even():
    """The 64-bit form that the GPU tests compare with: hand values, nearest
    representable by construction, ties on the even code."""
    from oracle import mx4_oracle as M
    u = np.array([0.0, 0.25, 0.26, 0.5, 0.74, 0.75, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 6.0, 7.9])
    want = np.array([0, 0, .5, .5, .5, 1, 1, 1.5, 2, 2, 3, 4, 4, 6, 6, 6])
    assert np.array_equal(M.MAGNITUDES[M.round_e2m1(u)], want)
    assert np.array_equal(M.round_e2m1(-u), M.round_e2m1(u) + 8)
    x = np.zeros((1, 64))
    x[0, 0], x[0, 40] = 7.0, 0.3
    code, s = M.quantize(x)
    assert s.tolist() == [[127, 127 - 4]] and M.values(code, s)[0, 0] == 6.0 and M.values(code, s)[0, 40] == 0.25
    rng = np.random.default_rng(0)
    v = rng.standard_normal((4, 96))
    r = M.rounded(v)
    step = np.ldexp(1.0, np.floor(np.log2(np.abs(v).reshape(4, 3, 32).max(-1))).astype(int) - 2).repeat(32, 1)
    grid = np.concatenate([-M.MAGNITUDES, M.MAGNITUDES])
    best = np.abs(v[..., None] - grid * step[..., None]).min(-1)
    assert np.allclose(np.abs(v - r), best, atol=0, rtol=1e-12)
