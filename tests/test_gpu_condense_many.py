"""luffy_condense on buckets of three to eight slots a token, over its kernels' sizes
(one block of slots, many, the fp8 screen), against the oracle."""
import numpy as np
import pytest

from oracle import block_oracle as B
from oracle import luffy_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_15419_amd as L
    L.load_library()


@pytest.mark.parametrize("dtype,T,d,E,k,cf", [
    ("bf16", 1, 64, 8, 8, 0.0), ("f32", 40, 64, 8, 8, 0.0), ("bf16", 333, 320, 3, 3, 0.0), ("f32", 900, 320, 6, 5, 1.0),
    ("bf16", 2000, 256, 16, 7, 0.6), ("f32", 1300, 192, 12, 4, 0.0), ("bf16", 1500, 2048, 8, 8, 0.0),
    ("bf16", 1400, 2112, 4, 3, 1.1)])
def test_condense(dtype, T, d, E, k, cf):
    import torch
    import paper_2411_15419_amd as L
    rng = np.random.default_rng(T + k)
    # centres in random directions, and tokens close to one each: no cosine near 0.8
    c = rng.standard_normal((max(1, T // 12), d))
    x = torch.from_numpy(c[rng.integers(0, len(c), T)] + 0.03 * rng.standard_normal((T, d)))
    x = x.to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    _, perm, off = B.buckets(idx, E, cf)
    C = L.capacity(T, k, E, cf)
    cap, S = (min(T, C) if C > 0 else T), len(perm)
    i32 = lambda n: torch.full((n,), -5, dtype=torch.int32, device="cuda")  # noqa: E731
    pt = i32(T * k)
    pt[:S] = torch.from_numpy(perm.astype(np.int32)).cuda()
    of, row, ro, tok, deg = i32(T * k), i32(T * k), i32(E + 1), i32(T * k), i32(T * k)
    x_rep = torch.full((T * k, d), -3.0, dtype=x.dtype, device="cuda")
    ws = torch.empty(L.condense_workspace_size(T, d, E, k, cap), dtype=torch.uint8, device="cuda")
    L.luffy_condense(x, pt, torch.from_numpy(off.astype(np.int32)).cuda(), k, cap, 0.8, of, row, ro, tok, x_rep, deg, ws)
    ref = O.condense(x.double().cpu().numpy(), perm, off, 0.8)
    assert np.array_equal(of[:S].cpu().numpy(), np.asarray(ref.rep_of_pos)[:S])
    assert np.array_equal(deg[:S].cpu().numpy(), np.asarray(ref.degree)[:S])
    assert np.array_equal(ro.cpu().numpy(), ref.rep_offsets)
    assert np.array_equal(row[:S].cpu().numpy(), np.asarray(ref.rep_row)[:S])
    R = int(ro[-1])
    assert 0 < R <= S and (R < S or T == 1)
    assert np.array_equal(tok[:R].cpu().numpy(), np.asarray(ref.rep_token)[:R])
    assert torch.equal(x_rep[:R], x[tok[:R].long()]) and bool((x_rep[R:] == -3.0).all())
