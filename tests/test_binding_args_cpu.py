"""What the binding of the 8-bit operators and of the layer for a few tokens lets through to the library, which sees addresses only: every tensor
with its type, size, contiguity and device.  No GPU: stand-ins for CUDA tensors and a library that counts its calls."""
import types

import pytest
import torch


class OnGpu:
    """A tensor that says it lives on a GPU."""

    def __init__(self, t, index=0):
        self.t, self.index, self.device = t, index, torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self.t, name)

    is_cuda = True

    def get_device(self):
        return self.index

    def transpose(self, a, b):
        return OnGpu(self.t.transpose(a, b), self.index)


@pytest.fixture
def B(monkeypatch):
    import __graft_entry__ as ge
    ge.build()
    from paper_2503_02495_b200 import binding
    calls = []
    names = ("uoe_fp8_quantize", "uoe_fp8_transpose", "uoe_fp8_gemm", "uoe_fp8_wgrad", "uoe_mlp_forward_fp8", "uoe_mlp_tokens")
    lib = types.SimpleNamespace(**{n: (lambda *a, n=n: calls.append(n) or 0) for n in names})
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    binding.calls = calls
    yield binding
    del binding.calls


F8, BF, F32, I32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32, torch.int32


def _t(*shape, dtype=BF, **kw):
    return OnGpu(torch.zeros(*shape, dtype=torch.uint8 if dtype is F8 else dtype).view(dtype), **kw)


def _spoil(args, name, how):
    """One argument of another kind: a tensor of another device, type or size, or one that is not contiguous."""
    v = args[name].t
    if how == "device":
        bad = OnGpu(v, 1)
    elif how == "host":
        bad = v
    elif how == "short":
        bad = OnGpu(v.flatten()[:-1])
    elif how == "type":
        bad = OnGpu(torch.zeros(v.shape, dtype=torch.float64))
    else:
        bad = OnGpu(torch.zeros((*v.shape, 2), dtype=torch.uint8 if v.dtype is F8 else v.dtype).view(v.dtype)[..., 0])
        if bad.is_contiguous():
            return None
    return dict(args, **{name: bad})


def _all_spoilt(B, call, args, skip=()):
    n = len(B.calls)
    call(args)
    assert len(B.calls) == n + 1
    for name in args:
        for how in ("device", "host", "short", "type", "strided"):
            if (name, how) in skip or (name == "ws" and how in ("short", "type")):
                continue                                            # (a short workspace is the library's to refuse)
            bad = _spoil(args, name, how)
            if bad is None:
                continue
            with pytest.raises(ValueError if how == "device" else AssertionError):
                call(bad)
            assert len(B.calls) == n + 1, (name, how)


def _routing(T, n, k, m, c):
    return dict(expert_idx=_t(T, k, dtype=I32), patch_idx=_t(T, k, c, dtype=I32), gate=_t(T, k, c, dtype=F32), p_samp=_t(T, n, dtype=F32),
                p_patch=_t(T, n, m, dtype=F32), expert_offsets=_t(n + 1, dtype=I32))


R = ("expert_idx", "patch_idx", "gate", "p_samp", "p_patch", "expert_offsets")


@pytest.mark.parametrize("weights", ["bf16", "f32", "fp8"])
def test_layer_for_a_few_tokens(B, weights):
    T, d, d_e, n, k = 3, 64, 40, 4, 2
    p = B.Problem(B=T, L=1, L_valid=1, d=d, n=n, k=k, m=1, c=1, d_e=d_e, dtype="f32" if weights == "f32" else "bf16")
    dt = p.torch_dtype
    args = dict(x=_t(T, 1, d, dtype=dt), W_r=_t(d, n, dtype=dt), b1=_t(n, d_e, dtype=dt), b2=_t(n, d, dtype=dt), y=_t(T, 1, d, dtype=dt),
                ws=_t(4096, dtype=torch.uint8), **_routing(T, n, k, 1, 1))
    if weights == "fp8":
        args.update(W1=_t(n, d_e, 128, dtype=F8), s1=_t(n, 1, 1, dtype=F32), W2=_t(n, d, 128, dtype=F8), s2=_t(n, 1, 1, dtype=F32))
    else:
        args.update(W1=_t(n, d, d_e, dtype=dt), W2=_t(n, d_e, d, dtype=dt))
    call = lambda a: B.uoe_mlp_tokens(p, *(a[q] for q in ("x", "W_r", "W1", "W2")), s1=a.get("s1"), s2=a.get("s2"), b1=a["b1"], b2=a["b2"],
                                      r=B.Routing(**{q: a[q] for q in R}), y=a["y"], ws=a["ws"], check=False)
    _all_spoilt(B, call, args)
    calls = len(B.calls)
    for q in R:                                                     # a set of outputs is complete or absent as a whole
        with pytest.raises(AssertionError):
            call(dict(args, **{q: None}))
    for q in ("W_r", "W1", "W2"):
        with pytest.raises(AssertionError):
            call(dict(args, **{q: None}))
    if weights == "fp8":
        for q in ("s1", "s2"):
            with pytest.raises(AssertionError):
                call(dict(args, **{q: None}))
    with pytest.raises(AssertionError):
        call(dict(args, y=_t(T - 1, 1, d, dtype=dt)))
    assert len(B.calls) == calls


def test_layer_on_8_bit_weights(B):
    p = B.Problem(B=2, L=64, L_valid=60, d=64, n=4, k=2, m=8, c=4, d_e=40)
    args = dict(x=_t(2, 64, 64), W1=_t(4, 40, 128, dtype=F8), s1=_t(4, 1, 1, dtype=F32), W2=_t(4, 64, 128, dtype=F8), s2=_t(4, 1, 1, dtype=F32),
                b1=_t(4, 40), b2=_t(4, 64), y=_t(2, 64, 64), ws=_t(4096, dtype=torch.uint8), **_routing(2, 4, 2, 8, 4))
    args = {q: v for q, v in args.items() if q not in ("p_samp", "p_patch")}
    call = lambda a: B.uoe_mlp_forward_fp8(p, *(a[q] for q in ("x", "W1", "s1", "W2", "s2")), B.Routing(**{q: a.get(q) for q in R}), b1=a["b1"], b2=a["b2"],
                                           y=a["y"], ws=a["ws"], check=False)
    _all_spoilt(B, call, args)
    n = len(B.calls)
    for q in ("W1", "s1", "W2", "s2", "expert_idx", "patch_idx", "gate", "expert_offsets"):
        with pytest.raises(AssertionError):
            call(dict(args, **{q: None}))
    assert len(B.calls) == n
    call(dict(args, b1=None, b2=None))


def test_products(B):
    p = B.Fp8Problem(n=2, M=256, N=40, K=100)
    args = dict(A=_t(256, 128, dtype=F8), sa=_t(1, 256, dtype=F32), W=_t(2, 40, 128, dtype=F8), sw=_t(2, 1, 1, dtype=F32), off=_t(3, dtype=I32),
                C=_t(256, 40), ws=_t(1024, dtype=torch.uint8))
    _all_spoilt(B, lambda a: B.uoe_fp8_gemm(p, *(a[q] for q in ("A", "sa", "W", "sw", "off")), C=a["C"], ws=a["ws"], check=False), args)
    p = B.Fp8Problem(n=2, M=64, N=40, K=256, dtype="f32")
    args = dict(A=_t(64, 256, dtype=F8), sa=_t(2, 64, dtype=F32), W=_t(40, 256, dtype=F8), sb=_t(2, 40, dtype=F32), off=_t(3, dtype=I32),
                dW=_t(2, 64, 40, dtype=F32), ws=_t(1024, dtype=torch.uint8))
    call = lambda a: B.uoe_fp8_wgrad(p, *(a[q] for q in ("A", "sa", "W", "sb", "off")), dW=a["dW"], ws=a["ws"], check=False)
    _all_spoilt(B, call, args)
    n = len(B.calls)
    for name, other in (("A", _t(256, 64, dtype=F8)), ("W", _t(256, 40, dtype=F8))):      # the other way round
        with pytest.raises(AssertionError):
            call(dict(args, **{name: other}))
    assert len(B.calls) == n


def test_quantisation(B):
    args = dict(x=_t(100, 60), q=_t(100, 128, dtype=F8), s=_t(1, 100, dtype=F32))
    _all_spoilt(B, lambda a: B.uoe_fp8_quantize(a["x"], "rows", q=a["q"], scale=a["s"]), args, skip=[("x", "short"), ("x", "strided")])
    with pytest.raises(AssertionError):
        B.uoe_fp8_quantize(OnGpu(torch.zeros(100, 60, 2, dtype=BF)[..., 0]), "rows")
    args = dict(x=_t(128, 60, dtype=F8), q=_t(60, 128, dtype=F8))
    _all_spoilt(B, lambda a: B.uoe_fp8_transpose(a["x"], q=a["q"]), args, skip=[("x", "short"), ("x", "strided")])
