"""What the serving entry points' binding refuses from the tensors alone (no GPU
needed: the checks come before anything is launched)."""
import pytest


def ffn_arguments():
    import torch
    u8 = dict(dtype=torch.uint8)
    E, d, d_ff, rows = 2, 64, 128, 4
    x = torch.zeros(6, d, dtype=torch.bfloat16)
    return dict(x=x, row_index=torch.zeros(rows, dtype=torch.int32), rep_offsets=torch.zeros(E + 1, dtype=torch.int32),
                w1q=torch.zeros(E, d_ff, d // 2, **u8), w1s=torch.zeros(E, 1, d_ff, 8, **u8),
                w2q=torch.zeros(E, d, d_ff // 2, **u8), w2s=torch.zeros(E, 1, d, 8, **u8), act="gelu", max_rows=rows,
                y_rep=torch.zeros(rows, d, dtype=torch.bfloat16), workspace=torch.zeros(1, **u8))


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    import paper_2411_15419_amd as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2411_15419_amd import build
        build.build()
    return L.load_library()


def test_expert_ffn_takes_32_bit_offsets_and_indices():
    """64-bit offsets (what a cumulative sum gives) and indices would be read as
    pairs of 32-bit ones."""
    import torch
    import paper_2411_15419_amd as L
    good = ffn_arguments()
    with pytest.raises(L.LuffyError, match="GPU"):          # nothing else is wrong with these
        L.luffy_mx4_expert_ffn(**good)
    with pytest.raises(L.LuffyError, match="rep_offsets must be int32"):
        L.luffy_mx4_expert_ffn(**dict(good, rep_offsets=good["rep_offsets"].long()))
    with pytest.raises(L.LuffyError, match="row_index must be int32"):
        L.luffy_mx4_expert_ffn(**dict(good, row_index=good["row_index"].long()))
    with pytest.raises(L.LuffyError, match="row_index must be int32"):
        L.luffy_mx4_expert_ffn(**dict(good, row_index=torch.zeros(3, dtype=torch.int32)))


def test_moe_few_refuses_misaligned_scales(lib):
    """Scales at an odd byte; 8-byte alignment is enough (the call then stops at
    its workspace, one byte short)."""
    import ctypes
    fake, eight, byte = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(257)
    need = lib.luffy_moe_few_workspace_size(4, 64, 4, 2, 128)

    def call(s1, s2):
        return lib.luffy_moe_few(fake, 4, 64, 1, fake, None, 4, 2, fake, s1, fake, s2, 2, 128, 0, fake, fake, fake,
                                 fake, need - 1, None)
    assert call(byte, fake) == -1 and b"aligned" in lib.luffy_last_error()
    assert call(fake, byte) == -1 and b"aligned" in lib.luffy_last_error()
    assert call(eight, eight) == -3
