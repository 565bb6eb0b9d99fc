"""Host-side checks of the 8-bit operators and of the layer for a few tokens that need no GPU: sizes, and refusals before any launch."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def uoe():
    import __graft_entry__ as ge
    ge.build()
    import paper_2503_02495_b200 as mod
    return mod


@pytest.fixture(scope="module")
def lib(uoe):
    lib = ctypes.CDLL(uoe.LIB_PATH)
    for name in ("uoe_fp8_quantize", "uoe_fp8_gemm", "uoe_fp8_wgrad", "uoe_mlp_forward_fp8", "uoe_mlp_tokens"):
        getattr(lib, name).restype = ctypes.c_int
    return lib


OK_PTR, ODD_PTR = ctypes.c_void_p(4096), ctypes.c_void_p(4104)        # never dereferenced: validation comes first
SZ = ctypes.c_size_t(1 << 40)


def test_quantize_refuses(lib):
    call = lambda G=1, R=4, C=4, dt=0, lay=0, x=OK_PTR, q=OK_PTR, s=OK_PTR: lib.uoe_fp8_quantize(G, R, C, dt, lay, x, q, s, None)
    for kw in (dict(G=0), dict(R=0), dict(C=-1), dict(dt=2), dict(lay=4), dict(lay=-1), dict(x=None), dict(q=None), dict(s=None), dict(x=ODD_PTR),
               dict(q=ODD_PTR), dict(s=ODD_PTR)):
        assert call(**kw) == 1, kw
    assert call(R=2147483647) == 2
    assert call(G=1 << 20, R=1 << 20, C=1 << 20, lay=2) == 2            # more tiles than a grid has CTAs
    assert call(G=1 << 20, R=1 << 20, C=1 << 20) == 2


def test_products_refuse(uoe, lib):
    for f in (lib.uoe_fp8_gemm, lib.uoe_fp8_wgrad):
        def call(n=2, M=256, N=64, K=128, dtype="f32", flags=0, ptr=(OK_PTR,) * 6, ws=OK_PTR, size=SZ):
            p = uoe.Fp8Problem(n=n, M=M, N=N, K=K, dtype=dtype).c_struct()
            p.flags = flags
            return f(ctypes.byref(p), *ptr, ws, size, None)
        for i in range(6):
            assert call(ptr=tuple(None if j == i else OK_PTR for j in range(6))) == 1, i      # the offsets too: there are two experts
            if i != 4:
                assert call(ptr=tuple(ODD_PTR if j == i else OK_PTR for j in range(6))) == 1, i
        for kw in (dict(n=0), dict(M=0), dict(N=0), dict(K=0), dict(flags=2), dict(ws=None), dict(ws=ODD_PTR)):
            assert call(**kw) == 1, kw
        assert call(n=33) == 2
        assert call(M=(1 << 30) + 1) == 2
        assert call(size=ctypes.c_size_t(16)) == 3
        assert f(None, *(OK_PTR,) * 6, OK_PTR, SZ, None) == 1
    p = uoe.Fp8Problem(n=1, M=4, N=4, K=4, dtype="bf16").c_struct()
    assert lib.uoe_fp8_wgrad(ctypes.byref(p), *(OK_PTR,) * 6, OK_PTR, SZ, None) == 2           # weight gradients are float32
    assert uoe.uoe_fp8_workspace_bytes(uoe.Fp8Problem(n=1, M=4, N=4, K=4)) >= 1024
    assert uoe.uoe_fp8_workspace_bytes(uoe.Fp8Problem(n=0, M=4, N=4, K=4)) == 0
    assert "power of two" in uoe.status_string(8)


def test_layer_on_8_bit_weights_refuses(uoe, lib):
    base = dict(B=2, L=64, L_valid=60, d=64, n=4, k=2, m=8, c=4, d_e=32)
    def call(kw=None, null=None, odd=None, size=SZ):
        p = uoe.Problem(**dict(base, **(kw or {}))).c_struct()
        args = [OK_PTR] * 13                # x W1 s1 W2 s2 b1 b2 expert_idx patch_idx gate offsets y ws
        if null is not None:
            args[null] = None
        if odd is not None:
            args[odd] = ODD_PTR
        return lib.uoe_mlp_forward_fp8(ctypes.byref(p), *args, size, None)
    for i in (0, 1, 2, 3, 4, 7, 8, 9, 10, 11, 12):
        assert call(null=i) == 1, i
    for i in (0, 1, 2, 3, 4, 5, 6, 11, 12):
        assert call(odd=i) == 1, i
    assert call(dict(d_e=0)) == 1 and call(dict(k=5)) == 1
    assert call(dict(dtype="f32")) == 2
    assert call(size=ctypes.c_size_t(1024)) == 3
    w = uoe.uoe_workspace_bytes(uoe.Problem(**base), uoe.UOE_OP_MLP_FWD_FP8)
    rows = uoe.uoe_max_routed_rows(uoe.Problem(**base))
    assert w >= rows * (128 + 128 + 2 * 64)
    assert uoe.uoe_workspace_bytes(uoe.Problem(**dict(base, dtype="f32")), uoe.UOE_OP_MLP_FWD_FP8) == 0


def test_layer_for_a_few_tokens_refuses(uoe, lib):
    base = dict(B=4, L=1, L_valid=1, d=64, n=4, k=2, m=1, c=1, d_e=32)
    def call(kw=None, args=None, size=SZ, r=None):
        p = uoe.Problem(**dict(base, **(kw or {}))).c_struct()
        a = dict(x=OK_PTR, Wr=OK_PTR, W1=OK_PTR, s1=None, W2=OK_PTR, s2=None, b1=None, b2=None)
        a.update(args or {})
        y, ws = a.pop("y", ctypes.c_void_p(8192)), a.pop("ws", OK_PTR)
        return lib.uoe_mlp_tokens(ctypes.byref(p), *a.values(), r, y, ws, size, None)
    for name in ("x", "Wr", "W1", "W2", "y", "ws"):
        assert call(args={name: None}) == 1, name
        assert call(args={name: ODD_PTR}) == 1, name
    assert call(args=dict(s1=OK_PTR)) == 1 and call(args=dict(s2=OK_PTR)) == 1      # one scale without the other
    assert call(args=dict(b1=ODD_PTR)) == 1 and call(args=dict(b2=ODD_PTR)) == 1
    assert call(args=dict(y=OK_PTR)) == 1                                             # in place
    assert call(dict(B=65)) == 2
    assert call(dict(L=2, L_valid=2)) == 2
    assert call(dict(L=2, L_valid=2, m=2, c=2)) == 2
    assert call(dict(d_e=12)) == 2                                                    # rows of 24 bytes
    assert call(dict(dtype="f32"), args=dict(s1=OK_PTR, s2=OK_PTR)) == 2
    assert call(size=ctypes.c_size_t(2048)) == 3
    from paper_2503_02495_b200 import binding as B
    r = B._Routing(4096, 4096, 4096, 4096, 4096, None)
    assert call(r=ctypes.byref(r)) == 1
    assert uoe.uoe_workspace_bytes(uoe.Problem(**base), uoe.UOE_OP_MLP_TOKENS) > 4 * 32 * 2
    assert uoe.uoe_workspace_bytes(uoe.Problem(**dict(base, B=65)), uoe.UOE_OP_MLP_TOKENS) == 0
    assert uoe.uoe_workspace_bytes(uoe.Problem(**dict(base, L=2, L_valid=2)), uoe.UOE_OP_MLP_TOKENS) == 0


def test_binding_checks_its_tensors(uoe):
    import torch
    with pytest.raises(AssertionError):
        uoe.uoe_fp8_quantize(torch.zeros(4, 4), "rows")                               # not on a GPU
    with pytest.raises(AssertionError):
        uoe.uoe_fp8_quantize(torch.zeros(4), "rows")
    with pytest.raises(AssertionError):
        uoe.uoe_fp8_quantize(torch.zeros(4, 4, dtype=torch.float16), "rows")
    with pytest.raises(ValueError):
        uoe.uoe_fp8_quantize(torch.zeros(4, 4), "columns")
