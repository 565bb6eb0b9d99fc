"""Host-side checks of uoe_fp8_transpose that need no GPU: refusals before any launch."""
import ctypes

import pytest

OK_PTR, ODD_PTR, OTHER = ctypes.c_void_p(4096), ctypes.c_void_p(4104), ctypes.c_void_p(8192)      # never dereferenced: validation comes first


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as ge
    ge.build()
    import paper_2503_02495_b200 as uoe
    lib = ctypes.CDLL(uoe.LIB_PATH)
    lib.uoe_fp8_transpose.restype = lib.uoe_fp8_quantize.restype = ctypes.c_int
    return lib


def test_transpose_refuses(lib):
    call = lambda G=1, R=128, C=4, x=OK_PTR, q=OTHER: lib.uoe_fp8_transpose(G, R, C, x, q, None)
    for kw in (dict(G=0), dict(R=0), dict(R=100), dict(C=0), dict(C=-5), dict(x=None), dict(q=None), dict(x=ODD_PTR), dict(q=ODD_PTR), dict(q=OK_PTR)):
        assert call(**kw) == 1, kw
    assert call(C=2147483647) == 2
    assert call(G=1 << 24, R=1 << 15) == 2                              # more tiles than a grid has CTAs
    assert call(G=(1 << 31) - 1, R=1 << 30, C=1 << 30) == 2
    assert call(R=1 << 30, C=1 << 20) == 2


def test_layout_of_an_operand_is_told_from_its_strides(monkeypatch):
    import torch
    from paper_2503_02495_b200 import binding as B
    seen = []
    monkeypatch.setattr(B, "uoe_fp8_transpose", lambda x: seen.append(tuple(x.shape)) or x.transpose(-1, -2).contiguous())
    q = torch.zeros(256, 77, dtype=torch.uint8)
    assert B._fp8_laid_out(q) is q and not seen
    assert B._fp8_laid_out(q.t()).is_contiguous() and seen == [(256, 77)]
    w = torch.zeros(3, 128, 40, dtype=torch.uint8)
    assert B._fp8_laid_out(w.transpose(1, 2)).is_contiguous() and seen[1:] == [(3, 128, 40)]
    cut = torch.zeros(77, 512, dtype=torch.uint8)[:, :256]                # neither: left for the check to refuse
    assert B._fp8_laid_out(cut) is cut and len(seen) == 2


@pytest.mark.parametrize("layout", [0, 1, 2, 3])
@pytest.mark.parametrize("sizes", [(1 << 30, 1 << 30, 1 << 30), ((1 << 31) - 1,) * 2 + (1 << 20,), (1 << 21, 1 << 30, 1 << 27)])
def test_quantise_refuses_what_no_grid_holds(lib, layout, sizes):
    """The number of CTAs is a product of three factors that passes 64 bits."""
    G, R, C = sizes
    assert lib.uoe_fp8_quantize(G, min(R, 0x7fffffff - 128), C, 0, layout, OK_PTR, OTHER, ctypes.c_void_p(1 << 20), None) == 2
