"""A block's entry points refuse bad arguments on the host, before anything is
enqueued, and the binding what it can see of the tensors (no GPU needed)."""
import ctypes
import math
import os

import pytest


@pytest.fixture(scope="module", autouse=True)
def lib():
    import paper_2411_15419_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2411_15419_amd import build
        build.build()
    return L.load_library()


FAKE = ctypes.c_void_p(256)     # never dereferenced: the checks fail first
ODD = ctypes.c_void_p(264)      # 8-byte aligned only
BYTE = ctypes.c_void_p(257)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def caller(fn, names, **good):
    names = names.split()
    assert set(good) <= set(names)

    def call(**change):
        assert set(change) <= set(names), set(change) - set(names)
        a = dict.fromkeys(names, FAKE)
        a.update(good)
        a.update(change)
        return fn(*(a[n] for n in names))
    return call


def norm_call(lib, **good):
    return caller(lib.luffy_block_norm, "x y T d dtype norm eps w_post b_post gate gate_kind res_scale w_pre b_pre o u "
                  "stream", **{**dict(T=4, d=64, dtype=1, norm=0, eps=1e-6, gate_kind=1, res_scale=1.0, stream=None),
                               **good})


def test_block_norm_refusals(lib):
    call = norm_call(lib)
    assert call(x=None) == INVALID and call(o=None) == INVALID and call(u=None) == INVALID
    assert call(y=None) == INVALID and call(w_pre=None) == INVALID
    for n in ("T", "d"):
        assert call(**{n: 0}) == INVALID and call(**{n: -5}) == INVALID
    assert call(dtype=2) == INVALID and call(norm=2) == INVALID and call(norm=-1) == INVALID
    assert call(eps=-1e-3) == INVALID and call(eps=math.nan) == INVALID and call(res_scale=math.nan) == INVALID
    assert call(gate_kind=3) == INVALID and call(gate_kind=0) == INVALID and call(gate=None) == INVALID
    assert call(w_post=None) == INVALID                            # b_post without it
    assert call(d=96) == UNSUPPORTED and call(d=32832) == UNSUPPORTED
    for n in ("x", "y", "w_post", "b_post", "gate", "w_pre", "b_pre", "o", "u"):
        assert call(**{n: ODD}) == INVALID, n
    # no layer's output: nothing that belongs to it
    alone = norm_call(lib, y=None, o=None, w_post=None, b_post=None, gate=None, gate_kind=0)
    assert alone(res_scale=0.5) == INVALID and alone(gate=FAKE, gate_kind=1) == INVALID
    assert alone(w_post=FAKE) == INVALID and alone(u=None, w_pre=None, b_pre=None) == INVALID
    assert norm_call(lib, w_pre=None, u=None)(b_pre=FAKE) == INVALID


def test_block_norm_backward_refusals(lib):
    call = caller(lib.luffy_block_norm_backward, "y o T d dtype norm eps w_post b_post gate gate_kind res_scale w_pre "
                  "dout du dx dy dgate dw_post db_post dw_pre db_pre workspace bytes stream", T=4, d=64, dtype=1, norm=1,
                  eps=1e-6, gate_kind=2, res_scale=1.0, bytes=1 << 30, stream=None)
    need = lib.luffy_block_norm_backward_workspace_size(4, 64)
    assert need > 0 and lib.luffy_block_norm_backward_workspace_size(0, 64) == 0
    assert call(dx=None) == INVALID and call(dout=None, du=None) == INVALID
    assert call(o=None) == INVALID and call(w_pre=None) == INVALID     # du needs both
    assert call(dy=None) == INVALID and call(y=None) == INVALID
    assert call(du=None) == INVALID                                    # dw_pre, db_pre of nothing
    assert call(w_post=None, b_post=None) == INVALID                   # dw_post of nothing
    assert call(gate=None, gate_kind=0) == INVALID                     # dgate of nothing
    assert call(T=0) == INVALID and call(d=100) == UNSUPPORTED and call(dtype=7) == INVALID
    for n in ("y", "o", "w_post", "b_post", "gate", "w_pre", "dout", "du", "dx", "dy", "dgate", "dw_post", "db_post",
              "dw_pre", "db_pre"):
        assert call(**{n: ODD}) == INVALID, n
    assert call(bytes=need - 1) == WORKSPACE and call(workspace=ODD) == WORKSPACE and call(workspace=None) == WORKSPACE
    assert call(T=2 ** 30 + 1) == UNSUPPORTED and norm_call(lib)(T=2 ** 31 - 1) == UNSUPPORTED


ROUTE = ("x T d dtype w_gate b_gate E k score balance groups top_groups group_best renormalise scale cf topk_idx "
         "topk_gate logits slot_pos perm_token offsets inv_norm workspace bytes stream")


def test_route_scored_refusals(lib):
    call = caller(lib.luffy_route_scored, ROUTE, T=8, d=64, dtype=1, E=16, k=4, score=1, groups=4, top_groups=2,
                  group_best=2, renormalise=1, scale=1.0, cf=0.0, bytes=1 << 20, stream=None)
    for n in ("x", "w_gate", "topk_idx", "topk_gate", "logits", "slot_pos", "perm_token", "offsets"):
        assert call(**{n: None}) == INVALID, n
    for n in ("T", "d", "E"):
        assert call(**{n: 0}) == INVALID
    assert call(k=0) == INVALID and call(k=17) == INVALID and call(dtype=3) == INVALID and call(score=2) == INVALID
    assert call(scale=math.inf) == INVALID and call(scale=math.nan) == INVALID
    assert call(groups=3) == INVALID and call(groups=0) == INVALID     # 16 experts
    assert call(top_groups=5) == INVALID and call(top_groups=0) == INVALID
    assert call(group_best=3) == INVALID and call(group_best=0) == INVALID
    assert call(groups=8, top_groups=1, k=3) == INVALID                # two experts are left
    assert call(E=65, groups=1, top_groups=1) == UNSUPPORTED and call(d=96) == UNSUPPORTED
    assert call(k=9, groups=1, top_groups=1) == UNSUPPORTED
    assert call(E=32, groups=32, top_groups=8) == UNSUPPORTED          # groups to choose from: 16 at most
    assert call(T=2 ** 30) == UNSUPPORTED and call(d=65536) == UNSUPPORTED
    assert call(T=2 ** 28 + 1, k=1) == UNSUPPORTED                     # grids count threads in 32 bits
    assert call(x=ODD) == INVALID and call(w_gate=ODD) == INVALID
    need = lib.luffy_route_workspace_size(8, 16, 4)
    assert call(bytes=need - 1) == WORKSPACE and call(workspace=ODD) == WORKSPACE


def test_route_scored_backward_refusals(lib):
    call = caller(lib.luffy_route_scored_backward, "x T d dtype w_gate E k score renormalise scale logits topk_idx "
                  "dgate dlogits dx_rep slot_pos rep_of_pos rep_row dx dw db workspace bytes stream", T=8, d=64, dtype=1,
                  E=16, k=4, score=1, renormalise=1, scale=1.0, bytes=1 << 30, stream=None)
    for n in ("x", "w_gate", "logits", "topk_idx", "dgate", "dx", "dw", "slot_pos", "rep_of_pos", "rep_row"):
        assert call(**{n: None}) == INVALID, n
    assert call(T=-1) == INVALID and call(k=17) == INVALID and call(score=5) == INVALID and call(dtype=2) == INVALID
    assert call(E=128) == UNSUPPORTED and call(d=32) == UNSUPPORTED and call(k=9) == UNSUPPORTED
    # 64 parts of T, each below 4 GiB
    assert call(T=64 * 66000, d=32768) == UNSUPPORTED and call(T=64 * 65000, d=32768, bytes=16) == WORKSPACE
    assert call(T=2 ** 28 + 1, k=1) == UNSUPPORTED
    for n in ("x", "w_gate", "dx_rep", "dx", "dw"):
        assert call(**{n: ODD}) == INVALID, n
    need = lib.luffy_route_scored_backward_workspace_size(8, 64, 16)
    assert need > 0 and lib.luffy_route_scored_backward_workspace_size(8, 64, 0) == 0
    assert call(bytes=need - 1) == WORKSPACE and call(workspace=None) == WORKSPACE


@pytest.mark.parametrize("name", ["quantize", "dequantize"])
def test_mx8_refusals(lib, name):
    fn = getattr(lib, "luffy_mx8_" + name)
    names = "x rows cols dtype q s stream" if name == "quantize" else "q s rows cols dtype x stream"
    call = caller(fn, names, rows=4, cols=64, dtype=0, stream=None)
    for n in ("x", "q", "s"):
        assert call(**{n: None}) == INVALID
    for n in ("rows", "cols"):
        assert call(**{n: 0}) == INVALID and call(**{n: -3}) == INVALID
    assert call(dtype=2) == INVALID and call(cols=48) == UNSUPPORTED and call(cols=32800) == UNSUPPORTED
    assert call(rows=2 ** 19 + 1, cols=32768) == UNSUPPORTED and call(rows=2 ** 31 - 1, cols=64) == UNSUPPORTED
    assert call(x=ODD) == INVALID and call(q=ODD) == INVALID and call(s=BYTE) == INVALID


def test_kept_ffn_refusals(lib):
    keep = caller(lib.luffy_expert_ffn_keep, "x row_index offsets E d d_ff w1 w2 act max_rows zq zs y workspace bytes "
                  "stream", E=4, d=64, d_ff=128, act=0, max_rows=8, bytes=1 << 40, stream=None)
    back = caller(lib.luffy_expert_ffn_backward_kept, "x x_scale x_rows row_index offsets E d d_ff w1 w2 act max_rows zq "
                  "zs dy dx dw1 dw2 dw_dtype workspace bytes stream", x_rows=8, E=4, d=64, d_ff=128, act=0, max_rows=8,
                  dw_dtype=1, bytes=1 << 40, stream=None)
    for n in ("x", "offsets", "w1", "w2", "zq", "zs"):
        assert keep(**{n: None}) == INVALID and back(**{n: None}) == INVALID, n
    assert keep(y=None) == INVALID
    for n in ("dy", "dx", "dw1", "dw2"):
        assert back(**{n: None}) == INVALID, n
    for call in (keep, back):
        assert call(E=0) == INVALID and call(max_rows=0) == INVALID and call(act=2) == INVALID
        assert call(E=65) == UNSUPPORTED and call(d=96) == UNSUPPORTED and call(d_ff=100) == UNSUPPORTED
        assert call(d_ff=32832) == UNSUPPORTED and call(max_rows=2 ** 25) == UNSUPPORTED
        assert call(zq=ODD) == INVALID and call(zs=BYTE) == INVALID and call(w1=ODD) == INVALID and call(x=ODD) == INVALID
    assert back(x_rows=0) == INVALID and back(x_scale=BYTE) == INVALID and back(dw_dtype=2) == INVALID
    assert back(dx=ODD) == INVALID and back(dw2=ODD) == INVALID
    need = lib.luffy_expert_ffn_backward_kept_workspace_size(8, 4, 64, 128)
    assert 0 < need < lib.luffy_expert_ffn_backward_workspace_size(8, 4, 64, 128, 1)
    assert back(bytes=need - 1) == WORKSPACE and back(workspace=ODD) == WORKSPACE
    assert keep(bytes=lib.luffy_expert_ffn_workspace_size(8, 4, 128, 1) - 1) == WORKSPACE
    assert lib.luffy_expert_ffn_backward_kept_workspace_size(0, 4, 64, 128) == 0


def test_combine_many_refusals(lib):
    call = caller(lib.luffy_combine_many, "y_rep rep_row slot_pos gate T k d dtype y stream", T=8, k=8, d=64, dtype=1,
                  stream=None)
    assert call(k=0) == INVALID and call(k=9) == INVALID and call(y=None) == INVALID and call(dtype=4) == INVALID
    assert call(d=96) == UNSUPPORTED and call(T=2 ** 28) == UNSUPPORTED
    back = caller(lib.luffy_combine_many_backward, "dy y_rep rep_row perm slot_pos gate offsets rep_offsets E T k d dtype "
                  "max_rows dy_rep dgate workspace bytes stream", E=4, T=8, k=8, d=64, dtype=1, max_rows=64,
                  bytes=1 << 30, stream=None)
    assert back(k=0) == INVALID and back(k=9) == INVALID and back(dy=None) == INVALID
    assert back(d=96) == UNSUPPORTED and back(bytes=16) == WORKSPACE
    # condensation takes as many choices, its history two
    condense = caller(lib.luffy_condense, "x T d dtype perm offsets E k max_bucket h of row ro tok x_rep degree inv "
                      "workspace bytes stream", T=8, d=64, dtype=1, E=16, max_bucket=8, h=0.9, x_rep=None, degree=None,
                      inv=None, bytes=16, stream=None)
    assert condense(k=8) == WORKSPACE and condense(k=9) == INVALID and condense(k=0) == INVALID


def test_binding_refusals():
    """Shapes, types and devices, from tensors on the host."""
    import torch
    import paper_2411_15419_amd as L
    T, d, E, k = 6, 64, 8, 3
    bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    x, v = torch.zeros(T, d, dtype=bf), torch.ones(d)
    good = dict(x=x, y=x, o=x.clone(), u=x.clone(), w_post=v, w_pre=v, gate=v)
    with pytest.raises(L.LuffyError, match="on the GPU"):          # nothing else is wrong with these
        L.luffy_block_norm(**good)
    for change, what in ((dict(y=x[:4]), "y must be"), (dict(o=x.float()), "o must be"), (dict(gate=v[:32]), "channel"),
                         (dict(gate=torch.zeros(T, d)), "token gate"), (dict(w_pre=v.to(bf)), "w_pre"),
                         (dict(x=x[0]), r"\[T, d\]"), (dict(norm="batch"), "norm")):
        with pytest.raises(L.LuffyError, match=what if "norm" not in change else "GPU|norm"):
            L.luffy_block_norm(**dict(good, **change))
    ws = torch.zeros(1, dtype=u8)
    with pytest.raises(L.LuffyError, match="dgate must be"):
        L.luffy_block_norm_backward(x, x, x, x, x.clone(), x.clone(), ws, gate=v, dgate=x)
    r = dict(x=x, w_gate=torch.zeros(E, d, dtype=bf), b_gate=None, k=k, score="sigmoid", capacity_factor=0.0,
             topk_idx=torch.zeros(T, k, dtype=i32), topk_gate=torch.zeros(T, k), logits=torch.zeros(T, E),
             slot_pos=torch.zeros(T, k, dtype=i32), perm_token=torch.zeros(T * k, dtype=i32),
             offsets=torch.zeros(E + 1, dtype=i32), workspace=ws)
    with pytest.raises(L.LuffyError, match="on the GPU"):
        L.luffy_route_scored(**r)
    for name, bad in (("topk_idx", r["topk_idx"].long()), ("topk_gate", r["topk_gate"][:, :2]),
                      ("logits", r["logits"].to(bf)), ("offsets", r["offsets"][:-1]), ("b_gate", torch.zeros(E, dtype=bf)),
                      ("perm_token", r["perm_token"][:-1])):
        with pytest.raises(L.LuffyError, match=name):
            L.luffy_route_scored(**dict(r, **{name: bad}))
    with pytest.raises(L.LuffyError, match="w_gate"):
        L.luffy_route_scored(**dict(r, w_gate=r["w_gate"].float()))
    g = dict(x=x, w_gate=r["w_gate"], score="sigmoid", logits=r["logits"], topk_idx=r["topk_idx"],
             dgate=r["topk_gate"], dx=x.clone(), dw_gate=torch.zeros(E, d), db_gate=None, workspace=ws)
    with pytest.raises(L.LuffyError, match="dx_rep must be"):
        L.luffy_route_scored_backward(**g, dx_rep=torch.zeros(T, d))
    with pytest.raises(L.LuffyError, match="rep_of_pos"):
        L.luffy_route_scored_backward(**g, dx_rep=x, slot_pos=r["slot_pos"], rep_of_pos=r["offsets"],
                                      rep_row=r["perm_token"])
    q, s = torch.zeros(T, d, dtype=torch.int8), torch.zeros(1, T, 8, dtype=u8)
    with pytest.raises(L.LuffyError, match="on the GPU"):
        L.luffy_mx8_quantize(x, q, s)
    with pytest.raises(L.LuffyError, match="int8"):
        L.luffy_mx8_quantize(x, q.to(u8), s)
    with pytest.raises(L.LuffyError, match="scales"):
        L.luffy_mx8_dequantize(q, s[:, :4], x)
    with pytest.raises(L.LuffyError, match="unsupported dtype"):
        L.luffy_mx8_quantize(x.half(), q, s)
    f = dict(x=x, row_index=None, rep_offsets=torch.zeros(3, dtype=i32), w1=torch.zeros(2, 128, d, dtype=bf),
             w2=torch.zeros(2, d, 128, dtype=bf), act="gelu", max_rows=T, zq=torch.zeros(T, 128, dtype=torch.int8),
             zs=s, y_rep=x.clone(), workspace=ws)
    with pytest.raises(L.LuffyError, match="on the GPU"):
        L.luffy_expert_ffn_keep(**f)
    for change, what in ((dict(zq=torch.zeros(T, 64, dtype=torch.int8)), "kept values"), (dict(max_rows=T + 1), "kept|rows"),
                         (dict(row_index=torch.zeros(T)), "row_index"), (dict(w2=f["w1"]), "w2"),
                         (dict(rep_offsets=f["rep_offsets"].long()), "rep_offsets"), (dict(y_rep=x[:4]), "y_rep"),
                         (dict(x=x.float()), "x must be"), (dict(act="tanh"), "act")):
        with pytest.raises(L.LuffyError, match=what):
            L.luffy_expert_ffn_keep(**dict(f, **change))
    for bad in (x.flatten(), x[0], x[None]):                       # one row is not as many as it has values
        with pytest.raises(L.LuffyError, match="x must be"):
            L.luffy_expert_ffn_keep(**dict(f, x=bad))
        with pytest.raises(L.LuffyError, match="x must be"):
            L.luffy_expert_ffn_backward_kept(bad, None, None, f["rep_offsets"], f["w1"], f["w2"], "gelu", T, f["zq"], s,
                                             x, x, f["w1"], f["w2"], ws)
    flat = r["slot_pos"].flatten()
    with pytest.raises(L.LuffyError, match="slot_pos"):
        L.luffy_combine_many(x, flat, flat, r["topk_gate"], x)
    with pytest.raises(L.LuffyError, match="slot_pos"):
        L.luffy_combine_many_backward(x, x, flat, flat, flat, r["topk_gate"], r["offsets"], r["offsets"], x,
                                      r["topk_gate"], ws)


def test_block_calls_in_another_order():
    """Calls that a block's documentation rules out, before anything is enqueued."""
    import torch
    import paper_2411_15419_amd as L

    def block(**more):
        b = L.MoEBlock.__new__(L.MoEBlock)
        b.__dict__.update(dict(T=4, d=64, dtype=torch.bfloat16, norm="rms", eps=1e-6, history=(0.1, 0.9)), **more)
        return b
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    a, b, other = block(), block(), block()
    for following in (a, block(norm="layer"), block(eps=1e-5)):
        with pytest.raises(L.LuffyError, match="share a pass"):
            a(x, following=following)
    with pytest.raises(L.LuffyError, match="of a call"):
        a.backward(x, x)                                           # none yet
    a.__dict__.update(normed=False, following=b, backed=False)
    for following in (None, other):
        with pytest.raises(L.LuffyError, match="the call had"):
            a.backward(x, x, following=following)
    for state in (dict(normed=True, backed=False), dict(normed=False, backed=True)):
        b.__dict__.update(following=None, **state)
        with pytest.raises(L.LuffyError, match="comes first"):
            a.backward(x, x, following=b)
    with pytest.raises(L.LuffyError, match="norms"):
        L.MoEStack([a, b])
