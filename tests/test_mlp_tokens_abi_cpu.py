"""Host-side check of the hidden widths that uoe_mlp_tokens takes; it needs no GPU: what is not refused reaches the last check, the workspace's size."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def uoe():
    import __graft_entry__ as ge
    ge.build()
    import paper_2503_02495_b200 as mod
    return mod


@pytest.mark.parametrize("dtype, scales, d_e, status", [("bf16", True, 33, 3), ("bf16", True, 12, 3), ("bf16", True, 1, 3), ("bf16", False, 12, 2),
                                                        ("bf16", False, 16, 3), ("f32", False, 6, 2), ("f32", False, 12, 3), ("f32", True, 8, 2)])
def test_hidden_widths(uoe, dtype, scales, d_e, status):
    lib = ctypes.CDLL(uoe.LIB_PATH)
    lib.uoe_mlp_tokens.restype = ctypes.c_int
    p = uoe.Problem(B=4, L=1, L_valid=1, d=64, n=4, k=2, m=1, c=1, d_e=d_e, dtype=dtype).c_struct()
    ok, y = ctypes.c_void_p(4096), ctypes.c_void_p(8192)             # never dereferenced: validation comes first
    s = ok if scales else None
    assert lib.uoe_mlp_tokens(ctypes.byref(p), ok, ok, ok, s, ok, s, None, None, None, y, ok, ctypes.c_size_t(2048), None) == status
