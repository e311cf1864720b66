"""Token-condensation MoE layer (Luffy, arXiv 2411.15419) on one MI355X.

Thin ctypes binding of ``libluffy.so`` (the HIP kernels behind the C ABI in
``include/luffy.h``).  Every function passes device pointers, sizes and the
current HIP stream through; every step of the layer runs in the library's
kernels.  torch supplies device memory and streams only.  There is no
fallback: without the built library every call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

__all__ = [
    "LuffyError", "load_library", "LUFFY_F32", "LUFFY_BF16", "LUFFY_ACT_GELU",
    "LUFFY_ACT_SILU", "luffy_route", "luffy_route_noalloc", "luffy_condense", "luffy_expert_ffn",
    "luffy_combine", "route_workspace_size", "condense_workspace_size",
    "expert_ffn_workspace_size", "capacity", "MoELayer", "LIB_PATH", "profile_kernel",
    "profile_read", "KERNELS", "adaptive_threshold", "AdaptiveThreshold",
    "luffy_combine_backward", "combine_backward_workspace_size", "luffy_expert_ffn_backward",
    "expert_ffn_backward_workspace_size", "luffy_condense_history", "history_size",
    "condense_history_workspace_size", "MoEStack", "CondensationDriver",
    "LUFFY_MX4", "FEW_MAX_TOKENS", "mx4_scale_bytes", "luffy_mx4_quantize", "luffy_mx4_dequantize",
    "luffy_mx4_matmul", "luffy_mx4_expert_ffn", "mx4_expert_ffn_workspace_size", "luffy_moe_few",
    "moe_few_workspace_size", "mx4_weights", "ServingLayer",
    "luffy_block_norm", "luffy_block_norm_backward", "block_norm_backward_workspace_size",
    "luffy_route_scored", "luffy_route_scored_backward", "route_scored_backward_workspace_size",
    "luffy_mx8_quantize", "luffy_mx8_dequantize", "luffy_expert_ffn_keep", "luffy_expert_ffn_backward_kept",
    "expert_ffn_backward_kept_workspace_size", "luffy_combine_many", "luffy_combine_many_backward", "MoEBlock",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libluffy.so")

LUFFY_F32, LUFFY_BF16, LUFFY_MX4 = 0, 1, 2
FEW_MAX_TOKENS = 64   # luffy_moe_few
LUFFY_ACT_GELU, LUFFY_ACT_SILU = 0, 1
_ACTS = {"gelu": LUFFY_ACT_GELU, "silu": LUFFY_ACT_SILU}
LUFFY_NORM_RMS, LUFFY_NORM_LAYER = 0, 1
_NORMS = {"rms": LUFFY_NORM_RMS, "layer": LUFFY_NORM_LAYER}
LUFFY_SCORE_SOFTMAX, LUFFY_SCORE_SIGMOID = 0, 1
_SCORES = {"softmax": LUFFY_SCORE_SOFTMAX, "sigmoid": LUFFY_SCORE_SIGMOID}
LUFFY_GATE_NONE, LUFFY_GATE_CHANNEL, LUFFY_GATE_TOKEN = 0, 1, 2

_c_int, _c_float, _c_size, _vp = ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p

_SIGS = {
    "luffy_abi_version": (_c_int, []),
    "luffy_status_string": (ctypes.c_char_p, [_c_int]),
    "luffy_last_error": (ctypes.c_char_p, []),
    "luffy_route_workspace_size": (_c_size, [_c_int, _c_int, _c_int]),
    "luffy_capacity": (_c_int, [_c_int, _c_int, _c_int, ctypes.c_double]),
    "luffy_route": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, ctypes.c_double,
                             _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_size, _vp]),
    "luffy_route_noalloc_max_bytes": (_c_size, []),
    "luffy_route_noalloc": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, ctypes.c_double,
                                     _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "luffy_condense_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "luffy_condense": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, _c_int,
                                _c_float, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_size, _vp]),
    "luffy_set_similarity_screen": (_c_int, [_c_int]),
    "luffy_similarity_screen_applies": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "luffy_history_size": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "luffy_condense_history_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "luffy_condense_history": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _vp, _c_int, _c_int, _c_int,
                                        _c_float, _vp, _vp, _c_float, _c_float, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _vp, _vp, _c_size, _vp]),
    "luffy_expert_ffn_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "luffy_expert_ffn": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp,
                                  _c_int, _c_int, _vp, _vp, _c_size, _vp]),
    "luffy_combine": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp]),
    "luffy_combine_many": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp]),
    "luffy_combine_many_backward": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _c_int,
                                             _c_int, _c_int, _c_int, _vp, _vp, _vp, _c_size, _vp]),
    "luffy_combine_backward_workspace_size": (_c_size, [_c_int, _c_int, _c_int]),
    "luffy_combine_backward": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _c_int,
                                        _c_int, _c_int, _c_int, _vp, _vp, _vp, _c_size, _vp]),
    "luffy_expert_ffn_backward_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "luffy_expert_ffn_backward": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp, _c_int,
                                           _c_int, _vp, _vp, _vp, _vp, _c_int, _vp, _c_size, _vp]),
    "luffy_mx4_scale_bytes": (_c_size, [_c_int, _c_int, _c_int]),
    "luffy_mx4_quantize": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp, _vp]),
    "luffy_mx4_dequantize": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _vp, _vp]),
    "luffy_mx4_matmul": (_c_int, [_vp, _vp, _c_int, _vp, _c_int, _c_int, _c_int, _vp, _vp, _vp, _c_int, _vp]),
    "luffy_mx4_expert_ffn_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "luffy_mx4_expert_ffn": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _vp, _vp, _vp, _vp, _c_int, _c_int, _vp,
                                      _vp, _c_size, _vp]),
    "luffy_moe_few_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "luffy_moe_few": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, _vp, _vp, _vp, _vp, _c_int,
                               _c_int, _c_int, _vp, _vp, _vp, _vp, _c_size, _vp]),
    "luffy_mx8_quantize": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _vp]),
    "luffy_mx8_dequantize": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _vp, _vp]),
    "luffy_expert_ffn_keep": (_c_int, [_vp, _vp, _vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, _vp, _vp, _vp,
                                       _vp, _c_size, _vp]),
    "luffy_expert_ffn_backward_kept_workspace_size": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "luffy_expert_ffn_backward_kept": (_c_int, [_vp, _vp, _c_int, _vp, _vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int,
                                                _c_int, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _vp, _c_size, _vp]),
    "luffy_route_scored": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _vp, _c_int, _c_int, _c_int, _vp, _c_int, _c_int,
                                    _c_int, _c_int, _c_float, ctypes.c_double, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                    _c_size, _vp]),
    "luffy_route_scored_backward_workspace_size": (_c_size, [_c_int, _c_int, _c_int]),
    "luffy_route_scored_backward": (_c_int, [_vp, _c_int, _c_int, _c_int, _vp, _c_int, _c_int, _c_int, _c_int, _c_float,
                                             _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_size,
                                             _vp]),
    "luffy_block_norm": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_float, _vp, _vp, _vp, _c_int, _c_float,
                                  _vp, _vp, _vp, _vp, _vp]),
    "luffy_block_norm_backward_workspace_size": (_c_size, [_c_int, _c_int]),
    "luffy_block_norm_backward": (_c_int, [_vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_float, _vp, _vp, _vp, _c_int,
                                           _c_float, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_size,
                                           _vp]),
    "luffy_adaptive_threshold": (_c_int, [ctypes.c_double, ctypes.c_double, ctypes.POINTER(ctypes.c_double)]),
    "luffy_profile_kernel": (_c_int, [ctypes.c_char_p]),
    "luffy_profile_read": (_c_int, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_c_int)]),
}

_LIB = None


class LuffyError(RuntimeError):
    pass


def load_library(path: str = LIB_PATH):
    """Loads libluffy.so once and declares the C signatures."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(path):
        raise LuffyError(f"{path} is not built; run `python -m paper_2411_15419_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        lib = load_library()
        msg = lib.luffy_last_error().decode()
        raise LuffyError(f"{what}: {lib.luffy_status_string(status).decode()} ({status}): {msg}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return LUFFY_F32
    if t.dtype == torch.bfloat16:
        return LUFFY_BF16
    raise LuffyError(f"unsupported dtype {t.dtype}")


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise LuffyError("tensor must be on the GPU")
    if not t.is_contiguous():
        raise LuffyError("tensor must be contiguous")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    # the current stream's handle without a Stream object: 0.3 us instead of
    # 2.7, of about 7 for a whole call (the tensors' checks came before: the
    # device is initialised)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def capacity(T: int, k: int, E: int, cf: float) -> int:
    """Per-expert capacity of luffy_route (luffy_capacity; 0 = unlimited)."""
    return int(load_library().luffy_capacity(int(T), int(k), int(E), float(cf)))


def route_workspace_size(T: int, E: int, k: int) -> int:
    return load_library().luffy_route_workspace_size(T, E, k)


def condense_workspace_size(T: int, d: int, E: int, k: int, max_bucket: int) -> int:
    return load_library().luffy_condense_workspace_size(T, d, E, k, max_bucket)


def set_similarity_screen(on: bool) -> bool:
    """Enables or disables the fp8 similarity screen of luffy_condense
    (luffy_set_similarity_screen); returns the previous setting."""
    return bool(load_library().luffy_set_similarity_screen(1 if on else 0))


def similarity_screen_applies(T: int, d: int, E: int, k: int, dtype: int = LUFFY_BF16) -> bool:
    """Whether a condense call of this shape takes the fp8 screen now."""
    return bool(load_library().luffy_similarity_screen_applies(int(T), int(d), int(E), int(k), int(dtype)))


def expert_ffn_workspace_size(max_rows: int, E: int, d_ff: int, dtype: int) -> int:
    return load_library().luffy_expert_ffn_workspace_size(max_rows, E, d_ff, dtype)


def luffy_route(x, w_gate, b_gate, k, capacity_factor, topk_idx, topk_gate, slot_pos,
                perm_token, offsets, workspace, stream=None, inv_norm=None):
    T, d = x.shape
    E = w_gate.shape[0]
    lib = load_library()
    _check(lib.luffy_route(_p(x), T, d, _dtype_code(x), _p(w_gate), _p(b_gate), E, k,
                           float(capacity_factor), _p(topk_idx), _p(topk_gate), _p(slot_pos),
                           _p(perm_token), _p(offsets), _p(inv_norm), _p(workspace),
                           workspace.numel(), _stream(stream)), "luffy_route")


def luffy_route_noalloc(x, w_gate, b_gate, k, capacity_factor, topk_idx, topk_gate, slot_pos,
                        perm_token, offsets, stream=None, inv_norm=None):
    """luffy_route without a workspace (the library's own scratch array;
    calls that may overlap on one GPU must be ordered by the caller)."""
    T, d = x.shape
    E = w_gate.shape[0]
    lib = load_library()
    _check(lib.luffy_route_noalloc(_p(x), T, d, _dtype_code(x), _p(w_gate), _p(b_gate), E, k,
                                   float(capacity_factor), _p(topk_idx), _p(topk_gate), _p(slot_pos),
                                   _p(perm_token), _p(offsets), _p(inv_norm), _stream(stream)),
           "luffy_route_noalloc")


def luffy_condense(x, perm_token, offsets, k, max_bucket, threshold, rep_of_pos, rep_row,
                   rep_offsets, rep_token, x_rep, degree, workspace, stream=None, inv_norm=None):
    T, d = x.shape
    E = offsets.numel() - 1
    lib = load_library()
    _check(lib.luffy_condense(_p(x), T, d, _dtype_code(x), _p(perm_token), _p(offsets), E, k,
                              max_bucket, float(threshold), _p(rep_of_pos), _p(rep_row),
                              _p(rep_offsets), _p(rep_token), _p(x_rep), _p(degree),
                              _p(inv_norm), _p(workspace), workspace.numel(), _stream(stream)),
           "luffy_condense")


def history_size(T: int, E: int, k: int, max_bucket: int) -> int:
    return int(load_library().luffy_history_size(T, E, k, max_bucket))


def condense_history_workspace_size(T: int, d: int, E: int, k: int, max_bucket: int) -> int:
    return int(load_library().luffy_condense_history_workspace_size(T, d, E, k, max_bucket))


def luffy_condense_history(x, perm_token, offsets, slot_pos, k, max_bucket, threshold, hist_in, hist_out, S1, S2,
                           rep_of_pos, rep_row, rep_offsets, rep_token, x_rep, degree, stats, workspace,
                           stream=None, inv_norm=None):
    """luffy_condense with the historical similarity of Sec. 5.1 step 2:
    hist_in is the previous block's record (or None), hist_out receives this
    block's (or None); stats (4 int64 or None) receives undecided pairs,
    decided pairs, tiles computed and tiles skipped."""
    T, d = x.shape
    E = offsets.numel() - 1
    _check(load_library().luffy_condense_history(
        _p(x), T, d, _dtype_code(x), _p(perm_token), _p(offsets), _p(slot_pos), E, k, max_bucket,
        float(threshold), _p(hist_in), _p(hist_out), float(S1), float(S2), _p(rep_of_pos), _p(rep_row),
        _p(rep_offsets), _p(rep_token), _p(x_rep), _p(degree), _p(inv_norm), _p(stats), _p(workspace),
        workspace.numel(), _stream(stream)), "luffy_condense_history")


def luffy_expert_ffn(x, row_index, rep_offsets, w1, w2, act, max_rows, y_rep, workspace,
                     stream=None):
    E, d_ff, d = w1.shape
    lib = load_library()
    act_code = _ACTS[act] if isinstance(act, str) else int(act)
    _check(lib.luffy_expert_ffn(_p(x), _p(row_index), _p(rep_offsets), E, d, d_ff,
                                _dtype_code(x), _p(w1), _p(w2), act_code, max_rows, _p(y_rep),
                                _p(workspace), workspace.numel(), _stream(stream)),
           "luffy_expert_ffn")


def luffy_combine(y_rep, rep_row, slot_pos, topk_gate, y, stream=None):
    T, k = slot_pos.shape
    d = y.shape[1]
    lib = load_library()
    _check(lib.luffy_combine(_p(y_rep), _p(rep_row), _p(slot_pos), _p(topk_gate), T, k, d,
                             _dtype_code(y), _p(y), _stream(stream)), "luffy_combine")


def combine_backward_workspace_size(T: int, k: int, max_rows: int) -> int:
    return int(load_library().luffy_combine_backward_workspace_size(T, k, max_rows))


def luffy_combine_backward(dy, y_rep, rep_row, perm_token, slot_pos, topk_gate, offsets, rep_offsets,
                           dy_rep, dgate, workspace, stream=None):
    """Transpose of luffy_combine: dy_rep (the representatives' rows) and
    dgate [T, k] from dy [T, d]."""
    T, d = dy.shape
    k = slot_pos.shape[1]
    max_rows = y_rep.shape[0]
    if dy_rep.shape != y_rep.shape or dy_rep.dtype != y_rep.dtype or dy.dtype != y_rep.dtype:
        raise LuffyError("dy, y_rep and dy_rep must share dtype; dy_rep must have y_rep's shape")
    E = rep_offsets.numel() - 1
    _check(load_library().luffy_combine_backward(
        _p(dy), _p(y_rep), _p(rep_row), _p(perm_token), _p(slot_pos), _p(topk_gate), _p(offsets),
        _p(rep_offsets), E, T, k, d, _dtype_code(dy), max_rows, _p(dy_rep), _p(dgate), _p(workspace),
        workspace.numel(), _stream(stream)),
        "luffy_combine_backward")


def expert_ffn_backward_workspace_size(max_rows: int, E: int, d: int, d_ff: int, dtype: int) -> int:
    return int(load_library().luffy_expert_ffn_backward_workspace_size(max_rows, E, d, d_ff, dtype))


def luffy_expert_ffn_backward(x, row_index, rep_offsets, w1, w2, act, max_rows, dy_rep, dx_rep, dw1, dw2,
                              workspace, stream=None):
    """Gradients of luffy_expert_ffn: dx_rep [max_rows, d] (bf16), dw1
    [E, d_ff, d] and dw2 [E, d, d_ff] (float32 or bf16, both the same) from
    dy_rep."""
    E, d_ff, d = w1.shape
    if dw1.dtype != dw2.dtype:
        raise LuffyError("luffy_expert_ffn_backward: dw1 and dw2 must have the same dtype")
    _check(load_library().luffy_expert_ffn_backward(
        _p(x), _p(row_index), _p(rep_offsets), E, d, d_ff, _dtype_code(x), _p(w1), _p(w2), _ACTS[act],
        max_rows, _p(dy_rep), _p(dx_rep), _p(dw1), _p(dw2), _dtype_code(dw1), _p(workspace), workspace.numel(),
        _stream(stream)), "luffy_expert_ffn_backward")


def mx4_scale_bytes(groups: int, rows: int, cols: int) -> int:
    """Bytes of the scales of a microscaled matrix [groups, rows, cols]."""
    return int(load_library().luffy_mx4_scale_bytes(int(groups), int(rows), int(cols)))


def _mx4_shape(q, s, what):
    """(groups, rows, cols) of a microscaled matrix, its tensors checked:
    values [groups, rows, cols/2] or [rows, cols/2], scales
    [(groups,) ceil(cols/256), rows, 8]."""
    if q.dtype != torch.uint8 or s.dtype != torch.uint8:
        raise LuffyError(f"{what}: values and scales must be uint8")
    if q.dim() not in (2, 3):
        raise LuffyError(f"{what}: values must be [rows, cols/2] or [groups, rows, cols/2]")
    groups, rows, cols = (q.shape[0] if q.dim() == 3 else 1), q.shape[-2], 2 * q.shape[-1]
    want = ((cols + 255) // 256, rows, 8)
    if tuple(s.shape) != ((groups,) + want if q.dim() == 3 else want):
        raise LuffyError(f"{what}: scales of values {tuple(q.shape)} must be "
                         f"{((groups,) + want if q.dim() == 3 else want)}, got {tuple(s.shape)}")
    return groups, rows, cols


def luffy_mx4_quantize(x, q, s, row_index=None, stream=None):
    """Rounds x [rows, cols] (or [groups, rows, cols]; float32 or bf16) to
    microscaled 4-bit values q [.., rows, cols/2] with scales s
    [.., ceil(cols/256), rows, 8] (uint8).  row_index (int32 [rows], 2-D q
    only): row r is x[row_index[r]]."""
    groups, rows, cols = _mx4_shape(q, s, "luffy_mx4_quantize")
    if x.shape[-1] != cols or x.dim() != q.dim() or (row_index is None and x.shape[:-1] != q.shape[:-1]):
        raise LuffyError(f"luffy_mx4_quantize: x {tuple(x.shape)} does not fit values {tuple(q.shape)}")
    if row_index is not None and (row_index.dtype != torch.int32 or row_index.numel() != rows):
        raise LuffyError("luffy_mx4_quantize: row_index must be int32 [rows]")
    _check(load_library().luffy_mx4_quantize(_p(x), _p(row_index), groups, rows, cols, _dtype_code(x), _p(q), _p(s),
                                             _stream(stream)), "luffy_mx4_quantize")


def mx4_weights(w, stream=None):
    """(values, scales) of weights w [groups, rows, cols] (float32 or bf16) in
    microscaled 4 bits, in tensors of their own."""
    groups, rows, cols = w.shape
    q = torch.empty(groups, rows, cols // 2, dtype=torch.uint8, device=w.device)
    s = torch.empty(groups, (cols + 255) // 256, rows, 8, dtype=torch.uint8, device=w.device)
    luffy_mx4_quantize(w, q, s, stream=stream)
    return q, s


def luffy_mx4_dequantize(q, s, x, stream=None):
    """The values of a microscaled matrix into x (float32 or bf16)."""
    groups, rows, cols = _mx4_shape(q, s, "luffy_mx4_dequantize")
    if tuple(x.shape) != tuple(q.shape[:-1]) + (cols,):
        raise LuffyError(f"luffy_mx4_dequantize: x {tuple(x.shape)} does not fit values {tuple(q.shape)}")
    _check(load_library().luffy_mx4_dequantize(_p(q), _p(s), groups, rows, cols, _dtype_code(x), _p(x),
                                               _stream(stream)), "luffy_mx4_dequantize")


def luffy_mx4_matmul(xq, xs, offsets, wq, ws, y, stream=None):
    """y[r] = W_e x_r on microscaled rows xq [M, K/2] and weights wq
    [E, N, K/2]; offsets (int32 [E+1]) buckets the rows by expert, None: one
    expert.  y [M, N] float32 or bf16."""
    _, M, K = _mx4_shape(xq, xs, "luffy_mx4_matmul")
    E, N, Kw = _mx4_shape(wq, ws, "luffy_mx4_matmul")
    if xq.dim() != 2 or wq.dim() != 3 or K != Kw or tuple(y.shape) != (M, N):
        raise LuffyError(f"luffy_mx4_matmul: rows {tuple(xq.shape)}, weights {tuple(wq.shape)}, y {tuple(y.shape)}")
    if offsets is not None and (offsets.dtype != torch.int32 or offsets.numel() != E + 1):
        raise LuffyError("luffy_mx4_matmul: offsets must be int32 [E + 1]")
    _check(load_library().luffy_mx4_matmul(_p(xq), _p(xs), M, _p(offsets), E, N, K, _p(wq), _p(ws), _p(y),
                                           _dtype_code(y), _stream(stream)), "luffy_mx4_matmul")


def mx4_expert_ffn_workspace_size(max_rows: int, E: int, d: int, d_ff: int) -> int:
    return int(load_library().luffy_mx4_expert_ffn_workspace_size(int(max_rows), int(E), int(d), int(d_ff)))


def luffy_mx4_expert_ffn(x, row_index, rep_offsets, w1q, w1s, w2q, w2s, act, max_rows, y_rep, workspace, stream=None):
    """luffy_expert_ffn on microscaled weights w1 [E, d_ff, d] and w2
    [E, d, d_ff]: the rows of x (bf16) and the hidden rows are rounded to 4 bits
    on the way."""
    E, d_ff, d = _mx4_shape(w1q, w1s, "luffy_mx4_expert_ffn")
    if _mx4_shape(w2q, w2s, "luffy_mx4_expert_ffn") != (E, d, d_ff):
        raise LuffyError(f"luffy_mx4_expert_ffn: weights {tuple(w1q.shape)} and {tuple(w2q.shape)}")
    if x.dtype != torch.bfloat16 or y_rep.dtype != torch.bfloat16 or x.shape[-1] != d or y_rep.shape[-1] != d:
        raise LuffyError("luffy_mx4_expert_ffn: x and y_rep must be bf16 rows of d values")
    if y_rep.shape[0] < max_rows or (row_index is None and x.shape[0] < max_rows) or rep_offsets.numel() != E + 1:
        raise LuffyError("luffy_mx4_expert_ffn: x, y_rep and rep_offsets do not fit max_rows and E")
    if rep_offsets.dtype != torch.int32:
        raise LuffyError("luffy_mx4_expert_ffn: rep_offsets must be int32 [E + 1]")
    if row_index is not None and (row_index.dtype != torch.int32 or row_index.numel() < max_rows):
        raise LuffyError("luffy_mx4_expert_ffn: row_index must be int32 [max_rows]")
    _check(load_library().luffy_mx4_expert_ffn(
        _p(x), _p(row_index), _p(rep_offsets), E, d, d_ff, _p(w1q), _p(w1s), _p(w2q), _p(w2s),
        _ACTS[act] if isinstance(act, str) else int(act), int(max_rows), _p(y_rep), _p(workspace), workspace.numel(),
        _stream(stream)), "luffy_mx4_expert_ffn")


def moe_few_workspace_size(T: int, d: int, E: int, k: int, d_ff: int) -> int:
    return int(load_library().luffy_moe_few_workspace_size(int(T), int(d), int(E), int(k), int(d_ff)))


def luffy_moe_few(x, w_gate, b_gate, w1, w2, k, act, topk_idx, topk_gate, y, workspace, w1_scale=None,
                  w2_scale=None, stream=None):
    """A whole layer (gate, top-k, expert FFN, combine; no condensation, no
    capacity) for T <= 64 tokens in one call.  Weights of x's dtype, or
    microscaled (uint8 values with their scales) under bf16 activations."""
    T, d = x.shape
    E = w_gate.shape[0]
    if w1_scale is not None or w2_scale is not None:
        if w1_scale is None or w2_scale is None:
            raise LuffyError("luffy_moe_few: microscaled weights need both scales")
        shape1, shape2 = _mx4_shape(w1, w1_scale, "luffy_moe_few"), _mx4_shape(w2, w2_scale, "luffy_moe_few")
        wtype = LUFFY_MX4
    else:
        shape1, shape2 = tuple(w1.shape), tuple(w2.shape)
        wtype = _dtype_code(w1)
        if w2.dtype != w1.dtype:
            raise LuffyError("luffy_moe_few: w1 and w2 must have the same dtype")
    if len(shape1) != 3 or shape1[0] != E or shape1[2] != d or shape2 != (E, d, shape1[1]) or w_gate.shape[1] != d:
        raise LuffyError(f"luffy_moe_few: w_gate {tuple(w_gate.shape)}, w1 {shape1}, w2 {shape2} for d = {d}")
    if w_gate.dtype != x.dtype or y.dtype != x.dtype or y.shape != x.shape:
        raise LuffyError("luffy_moe_few: w_gate and y must have x's dtype, y its shape")
    if b_gate is not None and (b_gate.dtype != torch.float32 or b_gate.numel() != E):
        raise LuffyError("luffy_moe_few: b_gate must be float32 [E]")
    if (topk_idx.dtype != torch.int32 or topk_gate.dtype != torch.float32 or topk_idx.numel() != T * k
            or topk_gate.numel() != T * k):
        raise LuffyError("luffy_moe_few: topk_idx must be int32 [T, k], topk_gate float32 [T, k]")
    _check(load_library().luffy_moe_few(
        _p(x), T, d, _dtype_code(x), _p(w_gate), _p(b_gate), E, k, _p(w1), _p(w1_scale), _p(w2), _p(w2_scale), wtype,
        shape1[1], _ACTS[act] if isinstance(act, str) else int(act), _p(topk_idx), _p(topk_gate), _p(y),
        _p(workspace), workspace.numel(), _stream(stream)), "luffy_moe_few")


def _named(table, value, what, name):
    if isinstance(value, str):
        if value not in table:
            raise LuffyError(f"{what}: {name} {value!r} is none of {', '.join(table)}")
        return table[value]
    return int(value)


def _fits(what, name, t, shape, dtype):
    """t (a tensor or None) has this shape and dtype."""
    if t is not None and (t.dtype != dtype or t.shape != shape):
        raise LuffyError(f"{what}: {name} must be {str(dtype)[6:]} {list(shape)}, got {str(t.dtype)[6:]} "
                         f"{list(t.shape)}")


def _device_ptrs(what, *tensors):
    """Pointers of contiguous tensors on the current device (None stays None):
    the launch goes to the current device's stream."""
    device, out = None, []
    for t in tensors:
        if t is not None:
            at = t.get_device()   # -1: not on a GPU
            if at != device:
                if at < 0:
                    raise LuffyError(f"{what}: tensor must be on the GPU")
                if device is None:
                    device = torch._C._cuda_getDevice()
                if at != device:
                    raise LuffyError(f"{what}: tensor on device {at}, the current one is {device}")
            if not t.is_contiguous():
                raise LuffyError(f"{what}: tensor must be contiguous")
            t = t.data_ptr()
        out.append(t)
    return out


def _block_gate(what, gate, T, d, dtype):
    """Kind of a block's gate: none, float32 [d], or [T, d] of dtype."""
    if gate is None:
        return LUFFY_GATE_NONE
    if gate.dim() == 1:
        _fits(what, "a channel gate", gate, (d,), torch.float32)
        return LUFFY_GATE_CHANNEL
    _fits(what, "a token gate", gate, (T, d), dtype)
    return LUFFY_GATE_TOKEN


def luffy_block_norm(x, y, o, u, *, norm="rms", eps=1e-6, res_scale=1.0, w_post=None, b_post=None, gate=None,
                     w_pre=None, b_pre=None, stream=None):
    """The residual stream around a layer: o = res_scale x + gate N(y; w_post,
    b_post) and u = N(o; w_pre, b_pre), rows [T, d] float32 or bf16, N the "rms"
    or "layer" norm.  y and o None: u of x.  w_pre and u None: o alone.  w_post
    None: y as it is.  gate: None, float32 [d], or [T, d] of x's dtype; weights
    and biases float32 [d]."""
    what = "luffy_block_norm"
    if x.dim() != 2:
        raise LuffyError(f"{what}: x must be [T, d], got {list(x.shape)}")
    shape, dtype, f32 = x.shape, x.dtype, torch.float32
    T, d = shape
    for name, t in (("y", y), ("o", o), ("u", u)):
        if t is not None and (t.shape != shape or t.dtype != dtype):
            _fits(what, name, t, shape, dtype)
    columns = (d,)
    for name, t in (("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("b_pre", b_pre)):
        if t is not None and (t.shape != columns or t.dtype != f32):
            _fits(what, name, t, columns, f32)
    kind = _block_gate(what, gate, T, d, dtype)
    dt = _dtype_code(x)
    x, y, w_post, b_post, gate, w_pre, b_pre, o, u = _device_ptrs(what, x, y, w_post, b_post, gate, w_pre, b_pre, o, u)
    _check(load_library().luffy_block_norm(x, y, T, d, dt, _named(_NORMS, norm, what, "norm"), eps, w_post, b_post, gate,
                                           kind, res_scale, w_pre, b_pre, o, u, _stream(stream)), what)


def block_norm_backward_workspace_size(T: int, d: int) -> int:
    return int(load_library().luffy_block_norm_backward_workspace_size(int(T), int(d)))


def luffy_block_norm_backward(y, o, dout, du, dx, dy, workspace, *, norm="rms", eps=1e-6, res_scale=1.0, w_post=None,
                              b_post=None, gate=None, w_pre=None, dgate=None, dw_post=None, db_post=None, dw_pre=None,
                              db_pre=None, stream=None):
    """Gradients of luffy_block_norm for dout = dL/do and du = dL/du (one of them
    may be None): dx, dy (None where y is), and those asked for of dgate (the
    gate's shape and dtype), dw_post, db_post, dw_pre and db_pre (float32 [d]).
    y, o, gate and weights as the forward had and left them."""
    what = "luffy_block_norm_backward"
    if dx.dim() != 2:
        raise LuffyError(f"{what}: dx must be [T, d], got {list(dx.shape)}")
    T, d = dx.shape
    for name, t in (("y", y), ("o", o), ("dout", dout), ("du", du), ("dy", dy)):
        _fits(what, name, t, dx.shape, dx.dtype)
    for name, t in (("w_post", w_post), ("b_post", b_post), ("w_pre", w_pre), ("dw_post", dw_post),
                    ("db_post", db_post), ("dw_pre", dw_pre), ("db_pre", db_pre)):
        _fits(what, name, t, (d,), torch.float32)
    kind = _block_gate(what, gate, T, d, dx.dtype)
    if gate is not None:
        _fits(what, "dgate", dgate, gate.shape, gate.dtype)
    dt, ws_bytes = _dtype_code(dx), workspace.numel() * workspace.element_size()
    (y, o, w_post, b_post, gate, w_pre, dout, du, dx, dy, dgate, dw_post, db_post, dw_pre, db_pre,
     workspace) = _device_ptrs(what, y, o, w_post, b_post, gate, w_pre, dout, du, dx, dy, dgate, dw_post, db_post,
                               dw_pre, db_pre, workspace)
    _check(load_library().luffy_block_norm_backward(
        y, o, T, d, dt, _named(_NORMS, norm, what, "norm"), eps, w_post, b_post, gate, kind, res_scale, w_pre, dout,
        du, dx, dy, dgate, dw_post, db_post, dw_pre, db_pre, workspace, ws_bytes, _stream(stream)), what)


def _mx8_shape(what, q, s):
    """(rows, cols) of a microscaled 8-bit matrix, its tensors checked: values
    int8 [rows, cols], scales uint8 [ceil(cols/256), rows, 8]."""
    if q.dim() != 2 or q.dtype != torch.int8:
        raise LuffyError(f"{what}: 8-bit values must be int8 [rows, cols], got {str(q.dtype)[6:]} {list(q.shape)}")
    rows, cols = q.shape
    _fits(what, "their scales", s, ((cols + 255) // 256, rows, 8), torch.uint8)
    return rows, cols


def luffy_mx8_quantize(x, q, s, stream=None):
    """Rounds x [rows, cols] (float32 or bf16) to microscaled 8-bit integers: int8
    values q [rows, cols] with scales s [ceil(cols/256), rows, 8] (uint8)."""
    what = "luffy_mx8_quantize"
    rows, cols = _mx8_shape(what, q, s)
    if x.shape != q.shape:
        raise LuffyError(f"{what}: x {list(x.shape)} does not fit values {list(q.shape)}")
    dt = _dtype_code(x)
    x, q, s = _device_ptrs(what, x, q, s)
    _check(load_library().luffy_mx8_quantize(x, rows, cols, dt, q, s, _stream(stream)), what)


def luffy_mx8_dequantize(q, s, x, stream=None):
    """The values of a microscaled 8-bit matrix into x (float32 or bf16)."""
    what = "luffy_mx8_dequantize"
    rows, cols = _mx8_shape(what, q, s)
    if x.shape != q.shape:
        raise LuffyError(f"{what}: x {list(x.shape)} does not fit values {list(q.shape)}")
    dt = _dtype_code(x)
    x, q, s = _device_ptrs(what, x, q, s)
    _check(load_library().luffy_mx8_dequantize(q, s, rows, cols, dt, x, _stream(stream)), what)


def _rows(what, name, t):
    """(rows, columns) of a bf16 matrix."""
    if t.dim() != 2 or t.dtype != torch.bfloat16:
        raise LuffyError(f"{what}: {name} must be bfloat16 [rows, cols], got {str(t.dtype)[6:]} {list(t.shape)}")
    return t.shape


def _ffn_shapes(what, x_rows, x_cols, row_index, rep_offsets, w1, w2, max_rows, zq, zs):
    """(E, d, d_ff), the tensors of an FFN that keeps Z checked."""
    bf, i32 = torch.bfloat16, torch.int32
    if w1.dim() != 3:
        raise LuffyError(f"{what}: w1 must be [E, d_ff, d], got {list(w1.shape)}")
    E, d_ff, d = w1.shape
    _fits(what, "w1", w1, (E, d_ff, d), bf)
    _fits(what, "w2", w2, (E, d, d_ff), bf)
    _fits(what, "rep_offsets", rep_offsets, (E + 1,), i32)
    if _mx8_shape(what, zq, zs) != (max_rows, d_ff):
        raise LuffyError(f"{what}: the kept values must be [{max_rows}, {d_ff}], got {list(zq.shape)}")
    if x_cols != d or (row_index is None and x_rows < max_rows):
        raise LuffyError(f"{what}: x [{x_rows}, {x_cols}] does not fit {max_rows} rows of {d}")
    if row_index is not None and (row_index.dtype != i32 or row_index.dim() != 1 or row_index.numel() < max_rows):
        raise LuffyError(f"{what}: row_index must be int32 [max_rows]")
    return E, d, d_ff


def luffy_expert_ffn_keep(x, row_index, rep_offsets, w1, w2, act, max_rows, zq, zs, y_rep, workspace, stream=None):
    """luffy_expert_ffn (bf16) that leaves its first product, before the
    activation, in microscaled 8 bits: zq int8 [max_rows, d_ff], zs uint8
    [ceil(d_ff/256), max_rows, 8], for luffy_expert_ffn_backward_kept.  Workspace:
    expert_ffn_workspace_size."""
    what = "luffy_expert_ffn_keep"
    x_rows, x_cols = _rows(what, "x", x)
    E, d, d_ff = _ffn_shapes(what, x_rows, x_cols, row_index, rep_offsets, w1, w2, max_rows, zq, zs)
    _fits(what, "y_rep", y_rep, (y_rep.shape[0], d), torch.bfloat16)
    if y_rep.shape[0] < max_rows:
        raise LuffyError(f"{what}: y_rep has {y_rep.shape[0]} rows of {max_rows}")
    ws_bytes, code = workspace.numel() * workspace.element_size(), _named(_ACTS, act, what, "act")
    x, row_index, rep_offsets, w1, w2, zq, zs, y_rep, workspace = _device_ptrs(
        what, x, row_index, rep_offsets, w1, w2, zq, zs, y_rep, workspace)
    _check(load_library().luffy_expert_ffn_keep(x, row_index, rep_offsets, E, d, d_ff, w1, w2, code, max_rows, zq, zs,
                                                y_rep, workspace, ws_bytes, _stream(stream)), what)


def expert_ffn_backward_kept_workspace_size(max_rows: int, E: int, d: int, d_ff: int) -> int:
    return int(load_library().luffy_expert_ffn_backward_kept_workspace_size(int(max_rows), int(E), int(d), int(d_ff)))


def luffy_expert_ffn_backward_kept(x, x_scale, row_index, rep_offsets, w1, w2, act, max_rows, zq, zs, dy_rep, dx_rep,
                                   dw1, dw2, workspace, stream=None):
    """luffy_expert_ffn_backward from luffy_expert_ffn_keep's zq, zs.  x: bf16 rows
    (x_scale None), or the int8 values of luffy_mx8_quantize with their scales;
    read through row_index where it is given."""
    what = "luffy_expert_ffn_backward_kept"
    bf = torch.bfloat16
    if x_scale is None:
        x_rows, x_cols = _rows(what, "x", x)
    else:
        x_rows, x_cols = _mx8_shape(what, x, x_scale)
    E, d, d_ff = _ffn_shapes(what, x_rows, x_cols, row_index, rep_offsets, w1, w2, max_rows, zq, zs)
    for name, t in (("dy_rep", dy_rep), ("dx_rep", dx_rep)):
        _fits(what, name, t, (t.shape[0], d), bf)
        if t.shape[0] < max_rows:
            raise LuffyError(f"{what}: {name} has {t.shape[0]} rows of {max_rows}")
    _fits(what, "dw1", dw1, w1.shape, dw1.dtype)
    _fits(what, "dw2", dw2, w2.shape, dw1.dtype)
    dw, code = _dtype_code(dw1), _named(_ACTS, act, what, "act")
    ws_bytes = workspace.numel() * workspace.element_size()
    x, x_scale, row_index, rep_offsets, w1, w2, zq, zs, dy_rep, dx_rep, dw1, dw2, workspace = _device_ptrs(
        what, x, x_scale, row_index, rep_offsets, w1, w2, zq, zs, dy_rep, dx_rep, dw1, dw2, workspace)
    _check(load_library().luffy_expert_ffn_backward_kept(
        x, x_scale, x_rows, row_index, rep_offsets, E, d, d_ff, w1, w2, code, max_rows, zq, zs, dy_rep, dx_rep, dw1,
        dw2, dw, workspace, ws_bytes, _stream(stream)), what)


def _router_shapes(what, x, w_gate):
    if x.dim() != 2 or w_gate.dim() != 2 or w_gate.shape[1] != x.shape[1] or w_gate.dtype != x.dtype:
        raise LuffyError(f"{what}: x [T, d] and w_gate [E, d] of one dtype, got {list(x.shape)} and "
                         f"{list(w_gate.shape)}")
    return x.shape[0], x.shape[1], w_gate.shape[0]


def luffy_route_scored(x, w_gate, b_gate, k, score, capacity_factor, topk_idx, topk_gate, logits, slot_pos, perm_token,
                       offsets, workspace, *, balance=None, groups=1, top_groups=1, group_best=1, renormalise=True,
                       scale=1.0, inv_norm=None, stream=None):
    """luffy_route with "softmax" or "sigmoid" scores, a bias for balance
    (float32 [E], in the choice alone), the experts of the top_groups best of
    `groups` groups, and up to 8 experts a token.  logits (float32 [T, E]) are what
    luffy_route_scored_backward needs."""
    what = "luffy_route_scored"
    T, d, E = _router_shapes(what, x, w_gate)
    f32, i32 = torch.float32, torch.int32
    _fits(what, "b_gate", b_gate, (E,), f32)
    _fits(what, "balance", balance, (E,), f32)
    _fits(what, "topk_idx", topk_idx, (T, k), i32)
    _fits(what, "topk_gate", topk_gate, (T, k), f32)
    _fits(what, "logits", logits, (T, E), f32)
    _fits(what, "slot_pos", slot_pos, (T, k), i32)
    _fits(what, "perm_token", perm_token, (T * k,), i32)
    _fits(what, "offsets", offsets, (E + 1,), i32)
    _fits(what, "inv_norm", inv_norm, (T,), f32)
    dt, ws_bytes = _dtype_code(x), workspace.numel() * workspace.element_size()
    (x, w_gate, b_gate, balance, topk_idx, topk_gate, logits, slot_pos, perm_token, offsets, inv_norm,
     workspace) = _device_ptrs(what, x, w_gate, b_gate, balance, topk_idx, topk_gate, logits, slot_pos, perm_token,
                               offsets, inv_norm, workspace)
    _check(load_library().luffy_route_scored(
        x, T, d, dt, w_gate, b_gate, E, k, _named(_SCORES, score, what, "score"), balance, groups, top_groups,
        group_best, bool(renormalise), scale, float(capacity_factor), topk_idx, topk_gate, logits, slot_pos,
        perm_token, offsets, inv_norm, workspace, ws_bytes, _stream(stream)), what)


def route_scored_backward_workspace_size(T: int, d: int, E: int) -> int:
    return int(load_library().luffy_route_scored_backward_workspace_size(int(T), int(d), int(E)))


def luffy_route_scored_backward(x, w_gate, score, logits, topk_idx, dgate, dx, dw_gate, db_gate, workspace, *,
                                renormalise=True, scale=1.0, dlogits=None, dx_rep=None, slot_pos=None,
                                rep_of_pos=None, rep_row=None, stream=None):
    """Gradients of luffy_route_scored's gates with its choices held fixed: dx
    [T, d], dw_gate [E, d] and db_gate [E] (float32; the last may be None) from
    dgate [T, k] and, where given, dlogits [T, E] of an auxiliary loss.  With
    dx_rep (and slot_pos, rep_of_pos, rep_row) the representatives' input
    gradients are added to their tokens' rows of dx."""
    what = "luffy_route_scored_backward"
    T, d, E = _router_shapes(what, x, w_gate)
    f32, i32 = torch.float32, torch.int32
    if topk_idx.dim() != 2:
        raise LuffyError(f"{what}: topk_idx must be [T, k], got {list(topk_idx.shape)}")
    k = topk_idx.shape[1]
    _fits(what, "topk_idx", topk_idx, (T, k), i32)
    _fits(what, "logits", logits, (T, E), f32)
    _fits(what, "dgate", dgate, (T, k), f32)
    _fits(what, "dlogits", dlogits, (T, E), f32)
    _fits(what, "dx", dx, x.shape, x.dtype)
    _fits(what, "dw_gate", dw_gate, (E, d), f32)
    _fits(what, "db_gate", db_gate, (E,), f32)
    if dx_rep is not None:
        if dx_rep.dim() != 2 or dx_rep.shape[1] != d or dx_rep.dtype != x.dtype:
            raise LuffyError(f"{what}: dx_rep must be rows of {d} values of x's dtype, got {list(dx_rep.shape)}")
        _fits(what, "slot_pos", slot_pos, (T, k), i32)
        _fits(what, "rep_of_pos", rep_of_pos, (T * k,), i32)
        _fits(what, "rep_row", rep_row, (T * k,), i32)
    dt, ws_bytes = _dtype_code(x), workspace.numel() * workspace.element_size()
    (x, w_gate, logits, topk_idx, dgate, dlogits, dx_rep, slot_pos, rep_of_pos, rep_row, dx, dw_gate, db_gate,
     workspace) = _device_ptrs(what, x, w_gate, logits, topk_idx, dgate, dlogits, dx_rep, slot_pos, rep_of_pos,
                               rep_row, dx, dw_gate, db_gate, workspace)
    _check(load_library().luffy_route_scored_backward(
        x, T, d, dt, w_gate, E, k, _named(_SCORES, score, what, "score"), bool(renormalise), scale, logits, topk_idx,
        dgate, dlogits, dx_rep, slot_pos, rep_of_pos, rep_row, dx, dw_gate, db_gate, workspace, ws_bytes,
        _stream(stream)), what)


def luffy_combine_many(y_rep, rep_row, slot_pos, topk_gate, y, stream=None):
    """luffy_combine for up to 8 slots a token."""
    what = "luffy_combine_many"
    if slot_pos.dim() != 2:
        raise LuffyError(f"{what}: slot_pos must be [T, k], got {list(slot_pos.shape)}")
    T, k = slot_pos.shape
    i32 = torch.int32
    if y.dim() != 2 or y_rep.dim() != 2 or y_rep.dtype != y.dtype or y_rep.shape[1] != y.shape[1]:
        raise LuffyError(f"{what}: y_rep {list(y_rep.shape)} and y {list(y.shape)} must be rows of one width and dtype")
    d = y.shape[1]
    _fits(what, "y", y, (T, d), y.dtype)
    _fits(what, "slot_pos", slot_pos, (T, k), i32)
    _fits(what, "topk_gate", topk_gate, (T, k), torch.float32)
    _fits(what, "rep_row", rep_row, (T * k,), i32)
    dt = _dtype_code(y)
    y_rep, rep_row, slot_pos, topk_gate, y = _device_ptrs(what, y_rep, rep_row, slot_pos, topk_gate, y)
    _check(load_library().luffy_combine_many(y_rep, rep_row, slot_pos, topk_gate, T, k, d, dt, y, _stream(stream)),
           what)


def luffy_combine_many_backward(dy, y_rep, rep_row, perm_token, slot_pos, topk_gate, offsets, rep_offsets, dy_rep,
                                dgate, workspace, stream=None):
    """luffy_combine_backward for up to 8 slots a token."""
    what = "luffy_combine_many_backward"
    if slot_pos.dim() != 2:
        raise LuffyError(f"{what}: slot_pos must be [T, k], got {list(slot_pos.shape)}")
    T, k = slot_pos.shape
    i32 = torch.int32
    if dy.dim() != 2 or y_rep.dim() != 2 or y_rep.shape[1] != dy.shape[1]:
        raise LuffyError(f"{what}: dy {list(dy.shape)} and y_rep {list(y_rep.shape)} must be rows of one width")
    d, E, max_rows = dy.shape[1], offsets.numel() - 1, y_rep.shape[0]
    _fits(what, "dy", dy, (T, d), y_rep.dtype)
    _fits(what, "dy_rep", dy_rep, y_rep.shape, y_rep.dtype)
    _fits(what, "slot_pos", slot_pos, (T, k), i32)
    for name, t in (("rep_row", rep_row), ("perm_token", perm_token)):
        _fits(what, name, t, (T * k,), i32)
    for name, t in (("topk_gate", topk_gate), ("dgate", dgate)):
        _fits(what, name, t, (T, k), torch.float32)
    for name, t in (("offsets", offsets), ("rep_offsets", rep_offsets)):
        _fits(what, name, t, (E + 1,), i32)
    dt, ws_bytes = _dtype_code(dy), workspace.numel() * workspace.element_size()
    (dy, y_rep, rep_row, perm_token, slot_pos, topk_gate, offsets, rep_offsets, dy_rep, dgate,
     workspace) = _device_ptrs(what, dy, y_rep, rep_row, perm_token, slot_pos, topk_gate, offsets, rep_offsets, dy_rep,
                               dgate, workspace)
    _check(load_library().luffy_combine_many_backward(
        dy, y_rep, rep_row, perm_token, slot_pos, topk_gate, offsets, rep_offsets, E, T, k, d, dt, max_rows, dy_rep,
        dgate, workspace, ws_bytes, _stream(stream)), what)


def adaptive_threshold(l_ini: float, l_prev: float) -> float:
    """h_t of Sec. 5.2 Eq. 2 from the first and the previous loss
    (luffy_adaptive_threshold)."""
    h = ctypes.c_double()
    _check(load_library().luffy_adaptive_threshold(float(l_ini), float(l_prev), ctypes.byref(h)),
           "luffy_adaptive_threshold")
    return h.value


class AdaptiveThreshold:
    """The threshold schedule of Sec. 5.2 over a training run: threshold()
    gives h_t for the coming iteration, record(loss) takes that iteration's
    loss.  The first recorded loss is l_ini; before any loss, and for the
    iteration after the first, h_t = 1/2."""

    def __init__(self):
        self.l_ini: Optional[float] = None
        self.l_prev: Optional[float] = None

    def threshold(self) -> float:
        if self.l_ini is None:
            return 0.5
        return adaptive_threshold(self.l_ini, self.l_prev)

    def record(self, loss: float) -> None:
        if self.l_ini is None:
            self.l_ini = float(loss)
        self.l_prev = float(loss)


def profile_kernel(name: Optional[str]) -> None:
    """Selects the kernel whose launches are bracketed by HIP events (None: off)."""
    _check(load_library().luffy_profile_kernel(name.encode() if name else None),
           "luffy_profile_kernel")


def profile_read():
    """(summed milliseconds, launches) of the selected kernel since the last read."""
    ms, n = ctypes.c_double(), _c_int()
    _check(load_library().luffy_profile_read(ctypes.byref(ms), ctypes.byref(n)),
           "luffy_profile_read")
    return ms.value, n.value


KERNELS = ("gate", "slot_scan", "slot_scatter", "norm", "gram", "gram_recheck", "greedy_round",
           "greedy_more", "greedy_finish", "rep_local", "rep_finalize", "gather", "ffn_queue", "ffn1", "ffn2",
           "ffn2_reduce", "combine")


def _on(stream):
    """What is allocated under it belongs to the stream that will use it."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _hold(t: torch.Tensor, raw) -> None:
    """t's memory stays t's until the stream of this handle is through with what it
    has been given so far."""
    if t.is_cuda:
        t.record_stream(torch.cuda.ExternalStream(raw, device=t.device) if raw else torch.cuda.default_stream(t.device))


def _workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator hands out 512-byte aligned blocks
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


@dataclass
class LayerBuffers:
    topk_idx: torch.Tensor
    topk_gate: torch.Tensor
    slot_pos: torch.Tensor
    perm_token: torch.Tensor
    offsets: torch.Tensor
    rep_of_pos: torch.Tensor
    rep_row: torch.Tensor
    rep_offsets: torch.Tensor
    rep_token: torch.Tensor
    degree: Optional[torch.Tensor]
    x_rep: Optional[torch.Tensor]
    y_rep: torch.Tensor
    y: torch.Tensor
    inv_norm: torch.Tensor
    ws_route: torch.Tensor
    ws_condense: torch.Tensor
    ws_ffn: torch.Tensor


class MoELayer:
    """Holds the weights and every buffer of one condensed MoE layer and runs
    the four library calls in order on the current stream.

    gather_x_rep=False (default) lets the FFN read representative rows of x
    through rep_token instead of materialising x_rep.
    """

    def __init__(self, w_gate, b_gate, w1, w2, *, k: int, act: str, threshold: float,
                 capacity_factor: float = 0.0, T: int, keep_degree: bool = True,
                 gather_x_rep: bool = False, norms_from_route: bool = True,
                 history: Optional[tuple] = None):
        self.w_gate, self.b_gate, self.w1, self.w2 = w_gate, b_gate, w1, w2
        self.k, self.act, self.h, self.cf = k, act, threshold, capacity_factor
        self.E, self.d_ff, self.d = w1.shape
        self.T = T
        self.norms_from_route = norms_from_route
        self.dtype = w1.dtype
        dev = w1.device
        S = T * k
        C = capacity(T, k, self.E, capacity_factor)
        self.max_bucket = min(T, C) if C > 0 else T
        # history = (S1, S2): condense with the historical similarity of the
        # previous block's record and leave this block's in self.record
        self.history = history
        i32 = dict(dtype=torch.int32, device=dev)
        self.buf = LayerBuffers(
            topk_idx=torch.empty(T, k, **i32),
            topk_gate=torch.empty(T, k, dtype=torch.float32, device=dev),
            slot_pos=torch.empty(T, k, **i32),
            perm_token=torch.empty(S, **i32),
            offsets=torch.empty(self.E + 1, **i32),
            rep_of_pos=torch.empty(S, **i32),
            rep_row=torch.empty(S, **i32),
            rep_offsets=torch.empty(self.E + 1, **i32),
            rep_token=torch.empty(S, **i32),
            degree=torch.empty(S, **i32) if keep_degree else None,
            x_rep=torch.empty(S, self.d, dtype=self.dtype, device=dev) if gather_x_rep else None,
            y_rep=torch.empty(S, self.d, dtype=self.dtype, device=dev),
            y=torch.empty(T, self.d, dtype=self.dtype, device=dev),
            inv_norm=torch.empty(T, dtype=torch.float32, device=dev),
            ws_route=_workspace(route_workspace_size(T, self.E, k), dev),
            ws_condense=_workspace((condense_history_workspace_size if history else condense_workspace_size)(
                T, self.d, self.E, k, self.max_bucket), dev),
            ws_ffn=_workspace(expert_ffn_workspace_size(
                S, self.E, self.d_ff, LUFFY_BF16 if self.dtype == torch.bfloat16 else LUFFY_F32),
                dev),
        )
        if history:
            self.record = _workspace(history_size(T, self.E, k, self.max_bucket), dev)
            self.hist_stats = torch.zeros(4, dtype=torch.int64, device=dev)

    def route(self, x, stream=None):
        b = self.buf
        luffy_route(x, self.w_gate, self.b_gate, self.k, self.cf, b.topk_idx, b.topk_gate,
                    b.slot_pos, b.perm_token, b.offsets, b.ws_route, stream, inv_norm=b.inv_norm)

    def condense(self, x, stream=None, threshold=None, hist_in=None):
        b = self.buf
        h = self.h if threshold is None else threshold
        inv = b.inv_norm if self.norms_from_route else None
        if self.history:
            S1, S2 = self.history
            luffy_condense_history(x, b.perm_token, b.offsets, b.slot_pos, self.k, self.max_bucket, h, hist_in,
                                   self.record, S1, S2, b.rep_of_pos, b.rep_row, b.rep_offsets, b.rep_token,
                                   b.x_rep, b.degree, self.hist_stats, b.ws_condense, stream, inv_norm=inv)
        else:
            if hist_in is not None:
                raise LuffyError("MoELayer: hist_in needs a layer built with history=(S1, S2)")
            luffy_condense(x, b.perm_token, b.offsets, self.k, self.max_bucket, h, b.rep_of_pos,
                           b.rep_row, b.rep_offsets, b.rep_token, b.x_rep, b.degree, b.ws_condense,
                           stream, inv_norm=inv)

    def expert_ffn(self, x, stream=None):
        b = self.buf
        if b.x_rep is not None:
            src, idx = b.x_rep, None
        else:
            src, idx = x, b.rep_token
        luffy_expert_ffn(src, idx, b.rep_offsets, self.w1, self.w2, self.act, self.T * self.k,
                         b.y_rep, b.ws_ffn, stream)

    def combine(self, stream=None):
        b = self.buf
        luffy_combine(b.y_rep, b.rep_row, b.slot_pos, b.topk_gate, b.y, stream)

    def backward(self, x, dy, stream=None, dw_dtype=torch.float32):
        """Gradients of the last call's output for dy = dL/dy [T, d], with its
        condensation held fixed (bf16 layers): returns (dgate [T, k] float32,
        dx_rep [T*k, d] with rows 0..R-1 the representatives' input
        gradients, in the order of rep_token, dw1, dw2 of dw_dtype: float32,
        or bfloat16 as the gradient of a bf16 parameter).  Buffers are
        allocated on the first call and reused."""
        b = self.buf
        if self.dtype != torch.bfloat16:
            raise LuffyError("MoELayer.backward: the expert FFN backward is bf16 only")
        S = self.T * self.k
        dev = dy.device
        if getattr(self, "_bwd", None) is None:
            E, dff, d = self.w1.shape
            with _on(stream):
                self._bwd = dict(
                    dy_rep=torch.empty_like(b.y_rep),
                    dgate=torch.empty(self.T, self.k, dtype=torch.float32, device=dev),
                    dx_rep=torch.empty(S, d, dtype=self.dtype, device=dev),
                    ws_c=_workspace(combine_backward_workspace_size(self.T, self.k, S), dev),
                    ws_f=_workspace(expert_ffn_backward_workspace_size(S, E, d, dff, LUFFY_BF16), dev),
                )
        g = self._bwd
        self._weight_gradients(g, dw_dtype, stream)
        luffy_combine_backward(dy, b.y_rep, b.rep_row, b.perm_token, b.slot_pos, b.topk_gate, b.offsets,
                               b.rep_offsets, g["dy_rep"], g["dgate"], g["ws_c"], stream)
        if b.x_rep is not None:
            src, idx = b.x_rep, None
        else:
            src, idx = x, b.rep_token
        luffy_expert_ffn_backward(src, idx, b.rep_offsets, self.w1, self.w2, self.act, S, g["dy_rep"],
                                  g["dx_rep"], g["dw1"], g["dw2"], g["ws_f"], stream)
        return g["dgate"], g["dx_rep"], g["dw1"], g["dw2"]

    def _weight_gradients(self, g, dw_dtype, stream):
        """dw1 and dw2 of dw_dtype in the backward's buffers g; those of another type
        go when the stream that wrote them has."""
        at, g["stream"] = g.get("stream"), _stream(stream) if self.w1.is_cuda else stream
        if "dw1" in g:
            if g["dw1"].dtype == dw_dtype:
                return
            for name in ("dw1", "dw2"):
                _hold(g[name], at)
        with _on(stream):
            for name, w in (("dw1", self.w1), ("dw2", self.w2)):
                g[name] = torch.empty(w.shape, dtype=dw_dtype, device=w.device)

    def __call__(self, x, stream=None, threshold=None, hist_in=None):
        if x.shape != (self.T, self.d) or x.dtype != self.dtype:
            raise LuffyError(f"x must be [{self.T}, {self.d}] {self.dtype}")
        self.route(x, stream)
        self.condense(x, stream, threshold, hist_in)
        self.expert_ffn(x, stream)
        self.combine(stream)
        return self.buf.y


class ServingLayer(MoELayer):
    """A layer that answers rather than learns.  __call__ runs T tokens (a
    prompt, a batch of prompts) through route, condense, expert FFN and combine;
    step runs up to FEW_MAX_TOKENS tokens (one of every stream being decoded)
    through luffy_moe_few, where condensation would find nothing to do.  A
    capacity_factor is for prompts alone: step never drops a token's expert.

    microscaled (default): the weights are rounded to microscaled 4 bits here,
    once, and only that form is kept (4.25 bits a weight); activations are bf16.
    """

    def __init__(self, w_gate, b_gate, w1, w2, *, microscaled: bool = True, **layer):
        super().__init__(w_gate, b_gate, w1, w2, **layer)
        if microscaled and self.dtype != torch.bfloat16:
            raise LuffyError("ServingLayer: microscaled weights take bf16 activations")
        dev = w1.device
        self.w1_scale = self.w2_scale = None
        if microscaled:
            self.w1, self.w1_scale = mx4_weights(w1)
            self.w2, self.w2_scale = mx4_weights(w2)
            self.buf.ws_ffn = _workspace(
                mx4_expert_ffn_workspace_size(self.T * self.k, self.E, self.d, self.d_ff), dev)
        n = FEW_MAX_TOKENS
        self.step_idx = torch.empty(n, self.k, dtype=torch.int32, device=dev)
        self.step_gate = torch.empty(n, self.k, dtype=torch.float32, device=dev)
        self.step_y = torch.empty(n, self.d, dtype=self.dtype, device=dev)
        self.ws_step = _workspace(moe_few_workspace_size(n, self.d, self.E, self.k, self.d_ff), dev)

    def expert_ffn(self, x, stream=None):
        if self.w1_scale is None:
            return super().expert_ffn(x, stream)
        b = self.buf
        src, idx = (x, b.rep_token) if b.x_rep is None else (b.x_rep, None)
        luffy_mx4_expert_ffn(src, idx, b.rep_offsets, self.w1, self.w1_scale, self.w2, self.w2_scale, self.act,
                             self.T * self.k, b.y_rep, self.buf.ws_ffn, stream)

    def backward(self, x, dy, stream=None, dw_dtype=torch.float32):
        raise LuffyError("ServingLayer has no backward")

    def step(self, x, stream=None):
        """y [n, d] of n <= FEW_MAX_TOKENS tokens x [n, d], valid until the next
        step; their experts and gates are step_idx[:n] and step_gate[:n]."""
        n = x.shape[0]
        if x.dim() != 2 or not 0 < n <= FEW_MAX_TOKENS:
            raise LuffyError(f"ServingLayer.step: x {tuple(x.shape)}, takes 1 to {FEW_MAX_TOKENS} tokens")
        y = self.step_y[:n]
        luffy_moe_few(x, self.w_gate, self.b_gate, self.w1, self.w2, self.k, self.act, self.step_idx[:n],
                      self.step_gate[:n], y, self.ws_step, w1_scale=self.w1_scale, w2_scale=self.w2_scale,
                      stream=stream)
        return y


class MoEBlock(MoELayer):
    """A layer that learns, with what stands around it (bf16):
        u = N(x; w_pre, b_pre),  y = the condensed layer of u,
        o = res_scale x + gate N(y; w_post, b_post)
    with the scored router (up to 8 experts a token).

    A block's last pass can be the next one's first: with `following` a call writes
    following.u beside o (one read of the stream), and following is then called
    with normed=True.  Buffers are allocated once; a block's outputs and gradients
    are valid until its next call.  A backward is of the last call, and refused where
    what it needs has been written over since.

    From its call to its backward a block keeps, of T tokens and S = T k slots: the
    experts' first product in microscaled 8 bits [S, d_ff], their outputs [S, d], y
    and o [T, d] in bf16, the logits and the choices; and u, in bf16 of its own or,
    with keep8, in microscaled 8 bits.  What it works with besides (u in bf16, the
    forward's and the backward's workspaces and gradients on their way) is its own
    too, unless it `shares` another block's: of blocks of the same sizes, called one
    after the other on one stream, all but the first then hold none of it.  Blocks
    that share are built with keep8 (the default with shares; the first one has to
    ask for it), as the next block's u takes the place of theirs; of no use without."""

    def __init__(self, w_gate, b_gate, w1, w2, *, w_pre, b_pre=None, w_post=None, b_post=None, gate=None,
                 res_scale: float = 1.0, norm: str = "rms", eps: float = 1e-6, score: str = "softmax", balance=None,
                 groups: int = 1, top_groups: int = 1, group_best: int = 1, renormalise: bool = True,
                 scale: float = 1.0, keep8: Optional[bool] = None, shares: Optional["MoEBlock"] = None, **layer):
        super().__init__(w_gate, b_gate, w1, w2, **layer)
        if self.dtype != torch.bfloat16:
            raise LuffyError("MoEBlock: the expert FFN backward is bf16 only")
        if self.history and self.k > 2:
            raise LuffyError("MoEBlock: historical similarity takes k <= 2")
        self.w_pre, self.b_pre, self.w_post, self.b_post, self.gate = w_pre, b_pre, w_post, b_post, gate
        self.res_scale, self.norm, self.eps = res_scale, norm, eps
        self.score, self.balance, self.renormalise, self.scale = score, balance, renormalise, scale
        self.keep8 = shares is not None if keep8 is None else keep8
        self.groups = dict(groups=groups, top_groups=top_groups, group_best=group_best)
        T, S, E, d, d_ff, dev = self.T, self.T * self.k, self.E, self.d, self.d_ff, w1.device
        bf = dict(dtype=torch.bfloat16, device=dev)

        def mx8(rows, cols):
            return (torch.empty(rows, cols, dtype=torch.int8, device=dev),
                    torch.empty((cols + 255) // 256, rows, 8, dtype=torch.uint8, device=dev))

        if self.buf.x_rep is not None:
            raise LuffyError("MoEBlock: gather_x_rep is of no use here")
        if shares is None:
            # what blocks can share; the backward's part comes with its first call
            self._work = dict(u=torch.empty(T, d, **bf))
            self._now = {}   # whose u and du the buffers hold: (block, the call before it or None), a call
        else:
            if not (shares.keep8 and self.keep8):
                raise LuffyError("MoEBlock: blocks that share keep u in 8 bits (keep8=True)")
            if shares._sizes() != self._sizes():
                raise LuffyError(f"MoEBlock: blocks that share are of the same sizes, not {shares._sizes()} and "
                                 f"{self._sizes()}")
            self._work, self._now = shares._work, shares._now
            for name in ("ws_route", "ws_condense", "ws_ffn"):
                setattr(self.buf, name, getattr(shares.buf, name))
        self.u, self.o = self._work["u"], torch.empty(T, d, **bf)
        self.logits = torch.empty(T, E, dtype=torch.float32, device=dev)
        self.zq, self.zs = mx8(S, d_ff)
        if self.keep8:
            self.uq, self.us = mx8(T, d)

    def _sizes(self):
        return dict(T=self.T, k=self.k, E=self.E, d=self.d, d_ff=self.d_ff, max_bucket=self.max_bucket,
                    history=self.history is not None, device=self.w1.device)

    def route(self, x, stream=None):
        b = self.buf
        luffy_route_scored(x, self.w_gate, self.b_gate, self.k, self.score, self.cf, b.topk_idx, b.topk_gate,
                           self.logits, b.slot_pos, b.perm_token, b.offsets, b.ws_route, balance=self.balance,
                           renormalise=self.renormalise, scale=self.scale, inv_norm=b.inv_norm, stream=stream,
                           **self.groups)

    def expert_ffn(self, x, stream=None):
        b = self.buf
        luffy_expert_ffn_keep(x, b.rep_token, b.rep_offsets, self.w1, self.w2, self.act, self.T * self.k, self.zq,
                              self.zs, b.y_rep, b.ws_ffn, stream)

    def combine(self, stream=None):
        b = self.buf
        luffy_combine_many(b.y_rep, b.rep_row, b.slot_pos, b.topk_gate, b.y, stream)

    def __call__(self, x, stream=None, threshold=None, hist_in=None, *, normed: bool = False, following=None):
        """o [T, d] for the stream x.  normed: self.u holds N(x) already (the call
        before this one had this block as its `following`)."""
        kw = dict(norm=self.norm, eps=self.eps, stream=stream)
        if x.shape != (self.T, self.d) or x.dtype != self.dtype:
            raise LuffyError(f"x must be [{self.T}, {self.d}] {self.dtype}")
        if following is not None and (following is self or (following.norm, following.eps) != (self.norm, self.eps)):
            raise LuffyError("MoEBlock: blocks that share a pass must be two, of the same norm and eps")
        made = self._now.get("u", (None, None))
        if normed and (made[0] is not self or made[1] is None):
            raise LuffyError("MoEBlock: normed=True, but self.u is not what a call with this block as its `following` "
                             "has left")
        self.normed, self.following, self.backed, self.call = normed, following, False, object()
        if not normed:
            made = self._now["u"] = (self, None)
            luffy_block_norm(x, None, None, self.u, w_pre=self.w_pre, b_pre=self.b_pre, **kw)
        self.made = made
        super().__call__(self.u, stream, threshold, hist_in)
        if self.keep8:
            luffy_mx8_quantize(self.u, self.uq, self.us, stream)
        luffy_block_norm(x, self.buf.y, self.o, following.u if following else None, res_scale=self.res_scale,
                         w_post=self.w_post, b_post=self.b_post, gate=self.gate,
                         w_pre=following.w_pre if following else None, b_pre=following.b_pre if following else None,
                         **kw)
        if following:
            following._now["u"] = (following, self.call)
        return self.o

    def _gradients(self, dw_dtype, stream=None):
        """Buffers of the backward, made on the first call."""
        if getattr(self, "_bwd", None) is None:
            with _on(stream):
                self._bwd = self._backward_buffers()
        self._weight_gradients(self._bwd, dw_dtype, stream)
        return self._bwd

    def _backward_buffers(self):
        T, S, E, d, d_ff, dev = self.T, self.T * self.k, self.E, self.d, self.d_ff, self.w1.device
        f32 = dict(dtype=torch.float32, device=dev)

        def vec(w):
            return None if w is None else torch.empty(d, **f32)

        rows = lambda n: torch.empty(n, d, dtype=torch.bfloat16, device=dev)  # noqa: E731
        if "du" not in self._work:
            self._work.update(
                dy=rows(T), du=rows(T), dy_rep=rows(S), dx_rep=rows(S), dlayer=torch.empty(T, self.k, **f32),
                ws_n=_workspace(block_norm_backward_workspace_size(T, d), dev),
                ws_c=_workspace(combine_backward_workspace_size(T, self.k, S), dev),
                ws_f=_workspace(expert_ffn_backward_kept_workspace_size(S, E, d, d_ff), dev),
                ws_r=_workspace(route_scored_backward_workspace_size(T, d, E), dev))
        return dict(
            self._work, dx=rows(T), dstream=rows(T), dw_gate=torch.empty(E, d, **f32), db_gate=torch.empty(E, **f32),
            dgate=None if self.gate is None else torch.empty_like(self.gate), dw_post=vec(self.w_post),
            db_post=vec(self.b_post), dw_pre=vec(self.w_pre), db_pre=vec(self.b_pre))

    def backward(self, x, dout, stream=None, dw_dtype=torch.float32, *, dlogits=None, following=None):
        """Gradients of the last call for dout = dL/do (bf16 [T, d]) and, where an
        auxiliary loss has one, dlogits (float32 [T, E]); the condensation and the
        choices are held fixed.  With the call's `following` its backward comes
        first, and dout is what it returned.  Returns (dx, gradients): a dict of
        dw1, dw2 (dw_dtype), dw_gate, db_gate, and dgate, dw_post, db_post, dw_pre,
        db_pre as far as the block has them; a block called with normed=True
        leaves dx and its dw_pre, db_pre to the block before it (dx is then the
        stream's gradient without the norm's share)."""
        if not hasattr(self, "backed") or following is not self.following:
            raise LuffyError("MoEBlock.backward: of a call, with the `following` that the call had")
        if following is not None:
            if not (following.backed and following.normed and following.made[1] is self.call):
                raise LuffyError("MoEBlock.backward: the following block, called with normed=True behind this call, "
                                 "comes first")
            if following._now["du"] is not following.call:
                raise LuffyError("MoEBlock.backward: the following block's gradient has been written over")
        if not self.keep8 and self._now["u"] is not self.made:
            raise LuffyError("MoEBlock.backward: u has been written over (keep8 keeps one of its own)")
        b, g = self.buf, self._gradients(dw_dtype, stream)
        kw = dict(norm=self.norm, eps=self.eps, stream=stream)
        S = self.T * self.k
        nxt = following._bwd if following is not None else {}
        luffy_block_norm_backward(b.y, self.o, dout, nxt.get("du"), g["dstream"], g["dy"], g["ws_n"],
                                  res_scale=self.res_scale, w_post=self.w_post, b_post=self.b_post, gate=self.gate,
                                  w_pre=following.w_pre if following else None, dgate=g["dgate"],
                                  dw_post=g["dw_post"], db_post=g["db_post"], dw_pre=nxt.get("dw_pre"),
                                  db_pre=nxt.get("db_pre"), **kw)
        luffy_combine_many_backward(g["dy"], b.y_rep, b.rep_row, b.perm_token, b.slot_pos, b.topk_gate, b.offsets,
                                    b.rep_offsets, g["dy_rep"], g["dlayer"], g["ws_c"], stream)
        u, us = (self.uq, self.us) if self.keep8 else (self.u, None)
        luffy_expert_ffn_backward_kept(u, us, b.rep_token, b.rep_offsets, self.w1, self.w2, self.act, S, self.zq,
                                       self.zs, g["dy_rep"], g["dx_rep"], g["dw1"], g["dw2"], g["ws_f"], stream)
        if self.keep8:
            self._now["u"] = (self, None)
            luffy_mx8_dequantize(self.uq, self.us, self.u, stream)
        self._now["du"] = self.call
        luffy_route_scored_backward(self.u, self.w_gate, self.score, self.logits, b.topk_idx, g["dlayer"], g["du"],
                                    g["dw_gate"], g["db_gate"], g["ws_r"], renormalise=self.renormalise,
                                    scale=self.scale, dlogits=dlogits, dx_rep=g["dx_rep"], slot_pos=b.slot_pos,
                                    rep_of_pos=b.rep_of_pos, rep_row=b.rep_row, stream=stream)
        dx = g["dstream"]
        if not self.normed:
            dx = g["dx"]
            luffy_block_norm_backward(None, x, g["dstream"], g["du"], dx, None, g["ws_n"], w_pre=self.w_pre,
                                      dw_pre=g["dw_pre"], db_pre=g["db_pre"], **kw)
        self.backed = True
        names = ("dw1", "dw2", "dw_gate", "db_gate", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
        return dx, {n: g[n] for n in names if g[n] is not None}


class MoEStack:
    """Consecutive MoE blocks over the same tokens, each condensing with the
    historical similarity of the block before it (Sec. 5.1 step 2): block b
    reads block b-1's record (block 0 computes every pair) and leaves its
    own.  Each block takes its own input (the caller's model computes block
    b's input from block b-1's output)."""

    def __init__(self, layers):
        if not layers or any(not L.history for L in layers):
            raise LuffyError("MoEStack: every layer needs history=(S1, S2)")
        if any(isinstance(L, MoEBlock) for L in layers):
            raise LuffyError("MoEStack: runs layers without their norms; call MoEBlocks one after the other")
        self.layers = list(layers)

    def __call__(self, xs, stream=None, threshold=None, ffn=True):
        """Runs every block on its input xs[b]; returns the blocks' outputs
        (with ffn=False only route and condense run, and nothing is
        returned)."""
        prev = None
        outs = []
        for layer, x in zip(self.layers, xs):
            layer.route(x, stream)
            layer.condense(x, stream, threshold, prev)
            if ffn:
                layer.expert_ffn(x, stream)
                layer.combine(stream)
                outs.append(layer.buf.y)
            prev = layer.record
        return outs if ffn else None


class CondensationDriver:
    """Training iterations over a stack of condensed MoE blocks with the
    adaptive threshold of Sec. 5.2 (Eq. 2): before an iteration, h_t comes
    from the first and the previous iteration's loss (AdaptiveThreshold; 1/2
    until a loss is recorded, as Eq. 2 gives for an unmoved loss); every
    block of the iteration condenses at h_t, each with the historical
    similarity of the block before it (Sec. 5.1 step 2); after it, the
    iteration's loss is recorded.  Eq. 2 as printed keeps h_t in
    (1/(1+e), 1/2] while the loss falls.

    stack: an MoEStack (or a single MoELayer, run alone)."""

    def __init__(self, stack, schedule: Optional[AdaptiveThreshold] = None):
        self.stack = stack
        self.schedule = schedule if schedule is not None else AdaptiveThreshold()
        self.thresholds = []
        self.losses = []

    def step(self, xs, loss, stream=None, ffn=True):
        """One iteration on the blocks' inputs xs (a list, one per block, or
        one tensor for a single layer).  loss: a number, or a callable that
        takes the outputs and returns this iteration's loss.  Returns
        (h_t, outputs)."""
        h = self.schedule.threshold()
        if isinstance(self.stack, MoEStack):
            outs = self.stack(xs, stream, threshold=h, ffn=ffn)
        else:
            outs = self.stack(xs, stream, threshold=h)
        value = float(loss(outs) if callable(loss) else loss)
        self.schedule.record(value)
        self.thresholds.append(h)
        self.losses.append(value)
        return h, outs
