"""ctypes binding of libuoe.so: argument marshalling only.

Every function here has the name and argument order of its C entry point (include/uoe.h), takes
torch CUDA tensors, allocates the outputs and the workspace with torch, passes raw pointers and the
current CUDA stream, and raises UoeError on a non-zero status.  No arithmetic of the method lives
in Python.  If the shared library is missing, importing this module fails: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libuoe.so")

UOE_ROW_ALIGN = 128
UOE_F32, UOE_BF16 = 0, 1
ACTS = {"gelu_erf": 0, "gelu_tanh": 1, "silu": 2, "identity": 3}
UOE_FLAG_RESIDUAL, UOE_FLAG_GATE, UOE_FLAG_CAUSAL, UOE_FLAG_DYNAMIC_C, UOE_FLAG_GENERAL_PATH = 1, 2, 4, 8, 16
UOE_OP_ROUTE, UOE_OP_MLP_FWD, UOE_OP_MLP_BWD, UOE_OP_SMHA_FWD, UOE_OP_SMHA_BWD = 0, 1, 2, 3, 4
UOE_OP_BALANCE_BWD, UOE_OP_MLP_FWD_FP8, UOE_OP_MLP_TOKENS = 5, 6, 7
UOE_FLAG_FP8_ANY_SCALE = 32
UOE_FP8_BLOCK, UOE_FP8_ANY_SCALE = 128, 1
FP8_LAYOUTS = {"rows": 0, "cols": 1, "blocks": 2, "blocks_t": 3}


class UoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class _Routing(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("expert_idx", "patch_idx", "gate", "p_samp", "p_patch", "expert_offsets")]


class _Problem(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in
                ("B", "L", "L_valid", "d", "n", "k", "m", "c", "d_e", "H", "d_h", "dtype", "act")] + \
               [("flags", ctypes.c_uint32), ("d_rope", ctypes.c_int32)]


class _Fp8Problem(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("n", "M", "N", "K", "dtype")] + [("flags", ctypes.c_uint32)]


class _Mirror:
    """A dataclass with a C struct: `ref` passes the struct, which is built again only when a field has changed."""

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_ref", None)

    @property
    def ref(self):
        ref = self.__dict__.get("_ref")
        if ref is None:
            ref = self.__dict__["_ref"] = ctypes.byref(self.c_struct())
        return ref

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_ref"}


@dataclass
class Fp8Problem(_Mirror):
    """Mirror of the C struct uoe_fp8_problem: a product of 8-bit operands (dtype: of the result)."""
    n: int
    M: int
    N: int
    K: int
    dtype: str = "bf16"
    any_scale: bool = False         # UOE_FP8_ANY_SCALE: scales that are not powers of two

    def c_struct(self) -> _Fp8Problem:
        return _Fp8Problem(self.n, self.M, self.N, self.K, UOE_BF16 if self.dtype == "bf16" else UOE_F32,
                           UOE_FP8_ANY_SCALE if self.any_scale else 0)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


@dataclass
class Problem(_Mirror):
    """Mirror of the C struct uoe_problem."""
    B: int
    L: int
    L_valid: int
    d: int
    n: int
    k: int
    m: int
    c: int
    d_e: int = 0
    H: int = 0
    d_h: int = 0
    dtype: str = "bf16"
    act: str = "silu"
    residual: bool = True
    gate: bool = True
    causal: bool = False
    dynamic_c: bool = False
    d_rope: int = 0
    general_path: bool = False      # UOE_FLAG_GENERAL_PATH: no single-mode shortcuts (same results)
    fp8_any_scale: bool = False     # UOE_FLAG_FP8_ANY_SCALE: 8-bit weights whose scales are not powers of two

    def c_struct(self) -> _Problem:
        flags = (UOE_FLAG_RESIDUAL if self.residual else 0) | (UOE_FLAG_GATE if self.gate else 0) | \
                (UOE_FLAG_CAUSAL if self.causal else 0) | (UOE_FLAG_DYNAMIC_C if self.dynamic_c else 0) | \
                (UOE_FLAG_GENERAL_PATH if self.general_path else 0) | (UOE_FLAG_FP8_ANY_SCALE if self.fp8_any_scale else 0)
        return _Problem(self.B, self.L, self.L_valid, self.d, self.n, self.k, self.m, self.c, self.d_e, self.H,
                        self.d_h, UOE_BF16 if self.dtype == "bf16" else UOE_F32, ACTS[self.act], flags, self.d_rope)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    @property
    def l_p(self) -> int:
        return self.L // self.m

    @property
    def l_a(self) -> int:
        return self.c * self.l_p


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2503_02495_b200/build.py` "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, i32p, f32p = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p
    pp = ctypes.POINTER(_Problem)
    lib.uoe_max_routed_rows.restype = ctypes.c_int64
    lib.uoe_max_routed_rows.argtypes = [pp]
    lib.uoe_workspace_bytes.restype = sz
    lib.uoe_workspace_bytes.argtypes = [pp, ctypes.c_int]
    lib.uoe_route.restype = ctypes.c_int
    lib.uoe_route.argtypes = [pp, vp, vp, i32p, i32p, f32p, f32p, f32p, i32p, vp, sz, vp]
    lib.uoe_route_static.restype = ctypes.c_int
    lib.uoe_route_static.argtypes = [pp, vp, vp, i32p, i32p, f32p, f32p, f32p, i32p, vp]
    lib.uoe_mlp_forward.restype = ctypes.c_int
    lib.uoe_mlp_forward.argtypes = [pp, vp, vp, vp, vp, vp, i32p, i32p, f32p, i32p, vp, vp, vp, sz, vp]
    lib.uoe_mlp_backward.restype = ctypes.c_int
    lib.uoe_mlp_backward.argtypes = [pp, vp, vp, vp, vp, i32p, i32p, f32p, i32p, f32p, f32p, vp, vp, vp, f32p, f32p,
                                     f32p, vp, sz, vp]
    lib.uoe_smha_forward.restype = ctypes.c_int
    lib.uoe_smha_forward.argtypes = [pp, vp, vp, vp, vp, vp, i32p, i32p, f32p, i32p, vp, f32p, vp, sz, vp]
    lib.uoe_smha_backward.restype = ctypes.c_int
    lib.uoe_smha_backward.argtypes = [pp, vp, vp, vp, vp, vp, vp, i32p, i32p, f32p, i32p, f32p, f32p, vp, vp, f32p, f32p,
                                      f32p, f32p, f32p, vp, sz, vp]
    lib.uoe_route_balance.restype = ctypes.c_int
    lib.uoe_route_balance.argtypes = [pp, f32p, ctypes.c_float, f32p, i32p, i32p, vp]
    lib.uoe_route_balance_backward.restype = ctypes.c_int
    lib.uoe_route_balance_backward.argtypes = [pp, vp, vp, f32p, ctypes.c_float, f32p, vp, f32p, vp, sz, vp]
    p8, i32 = ctypes.POINTER(_Fp8Problem), ctypes.c_int32
    lib.uoe_fp8_quantize.restype = ctypes.c_int
    lib.uoe_fp8_quantize.argtypes = [i32, i32, i32, i32, i32, vp, vp, f32p, vp]
    lib.uoe_fp8_transpose.restype = ctypes.c_int
    lib.uoe_fp8_transpose.argtypes = [i32, i32, i32, vp, vp, vp]
    lib.uoe_fp8_workspace_bytes.restype = sz
    lib.uoe_fp8_workspace_bytes.argtypes = [p8]
    for f in (lib.uoe_fp8_gemm, lib.uoe_fp8_wgrad):
        f.restype = ctypes.c_int
        f.argtypes = [p8, vp, f32p, vp, f32p, i32p, vp, vp, sz, vp]
    lib.uoe_mlp_forward_fp8.restype = ctypes.c_int
    lib.uoe_mlp_forward_fp8.argtypes = [pp, vp, vp, f32p, vp, f32p, vp, vp, i32p, i32p, f32p, i32p, vp, vp, sz, vp]
    lib.uoe_mlp_tokens.restype = ctypes.c_int
    lib.uoe_mlp_tokens.argtypes = [pp, vp, vp, vp, f32p, vp, f32p, vp, vp, ctypes.POINTER(_Routing), vp, vp, sz, vp]
    lib.uoe_block_workspace_bytes.restype = sz
    lib.uoe_block_workspace_bytes.argtypes = [pp, pp]
    lib.uoe_block_forward.restype = ctypes.c_int
    lib.uoe_block_forward.argtypes = [pp, pp] + [vp] * 9 + [ctypes.POINTER(_Routing)] * 2 + [vp, vp, vp, f32p, vp, sz, vp]
    lib.uoe_status_string.restype = ctypes.c_char_p
    lib.uoe_status_string.argtypes = [ctypes.c_int]
    lib.uoe_workspace_init.restype = ctypes.c_int
    lib.uoe_workspace_init.argtypes = [vp, sz, vp]
    lib.uoe_read_device_status.restype = ctypes.c_int
    lib.uoe_read_device_status.argtypes = [vp, vp]
    lib.uoe_launch_count.restype = ctypes.c_int64
    lib.uoe_launch_count.argtypes = []
    lib.uoe_tensor_map_encodings.restype = ctypes.c_int64
    lib.uoe_tensor_map_encodings.argtypes = []
    lib.uoe_profile_enable.restype = None
    lib.uoe_profile_enable.argtypes = [ctypes.c_int]
    lib.uoe_profile_count.restype = ctypes.c_int
    lib.uoe_profile_count.argtypes = []
    lib.uoe_profile_get.restype = ctypes.c_int
    lib.uoe_profile_get.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float)]
    return lib


_lib = _load()


def status_string(status: int) -> str:
    return _lib.uoe_status_string(int(status)).decode()


def _ptr(t):
    return None if t is None else t.data_ptr()


# (torch.cuda.current_stream() builds a Stream object, 6 us of a call that enqueues in 12)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(st: int, where: str):
    if st != 0:
        raise UoeError(st, where)


def _contig(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors must be contiguous CUDA tensors"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return t


def uoe_max_routed_rows(prob: Problem) -> int:
    return int(_lib.uoe_max_routed_rows(ctypes.byref(prob.c_struct())))


def uoe_workspace_bytes(prob: Problem, op: int) -> int:
    return int(_lib.uoe_workspace_bytes(ctypes.byref(prob.c_struct()), op))


def uoe_launch_count() -> int:
    return int(_lib.uoe_launch_count())


def uoe_tensor_map_encodings() -> int:
    return int(_lib.uoe_tensor_map_encodings())


def uoe_profile_enable(on: bool) -> None:
    _lib.uoe_profile_enable(1 if on else 0)


def uoe_profile_records():
    """[(label, milliseconds)] of every launch recorded since uoe_profile_enable(True)."""
    out = []
    for i in range(_lib.uoe_profile_count()):
        name, ms = ctypes.c_char_p(), ctypes.c_float()
        _check(_lib.uoe_profile_get(i, ctypes.byref(name), ctypes.byref(ms)), "uoe_profile_get")
        out.append((name.value.decode(), float(ms.value)))
    return out


def alloc_workspace(prob: Problem, op: int, device="cuda") -> torch.Tensor:
    nbytes = uoe_workspace_bytes(prob, op)
    if nbytes == 0:
        raise UoeError(1, "uoe_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        _check(_lib.uoe_workspace_init(_ptr(ws), nbytes, _stream()), "uoe_workspace_init")
    return ws


def uoe_read_device_status(ws: torch.Tensor) -> int:
    return int(_lib.uoe_read_device_status(_ptr(ws), _stream()))


@dataclass
class Routing:
    expert_idx: torch.Tensor      # [B,k] int32
    patch_idx: torch.Tensor       # [B,k,c] int32
    gate: torch.Tensor            # [B,k,c] float32
    p_samp: torch.Tensor          # [B,n] float32
    p_patch: torch.Tensor         # [B,n,m] float32
    expert_offsets: torch.Tensor  # [n+1] int32


def alloc_routing(prob: Problem, device="cuda") -> Routing:
    i32, f32 = torch.int32, torch.float32
    return Routing(torch.empty(prob.B, prob.k, dtype=i32, device=device),
                   torch.empty(prob.B, prob.k, prob.c, dtype=i32, device=device),
                   torch.empty(prob.B, prob.k, prob.c, dtype=f32, device=device),
                   torch.empty(prob.B, prob.n, dtype=f32, device=device),
                   torch.empty(prob.B, prob.n, prob.m, dtype=f32, device=device),
                   torch.empty(prob.n + 1, dtype=i32, device=device))


def uoe_route(prob: Problem, x, W_r, out: Routing | None = None, ws=None, check: bool = True) -> Routing:
    _contig(x, prob.torch_dtype)
    _contig(W_r, prob.torch_dtype)
    r = out if out is not None else alloc_routing(prob, x.device)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_ROUTE, x.device)
    st = _lib.uoe_route(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(W_r), _ptr(r.expert_idx), _ptr(r.patch_idx),
                        _ptr(r.gate), _ptr(r.p_samp), _ptr(r.p_patch), _ptr(r.expert_offsets), _ptr(ws), ws.numel(),
                        _stream())
    _check(st, "uoe_route")
    if check:
        _check(uoe_read_device_status(ws), "uoe_route (device)")
    return r


UOE_ROUTE_STATIC_SCRATCH_BYTES = 2 << 20


def uoe_route_static(prob: Problem, x, W_r, out: Routing | None = None) -> Routing:
    """uoe_route for callers that cannot supply a workspace: the scratch is a fixed array inside the
    library (limit UOE_ROUTE_STATIC_SCRATCH_BYTES).  Only the output tensors are created here, and only
    when `out` is not given; the C call itself allocates nothing.  Calls on one device must not overlap."""
    _contig(x, prob.torch_dtype)
    _contig(W_r, prob.torch_dtype)
    r = out if out is not None else alloc_routing(prob, x.device)
    st = _lib.uoe_route_static(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(W_r), _ptr(r.expert_idx),
                               _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.p_samp), _ptr(r.p_patch),
                               _ptr(r.expert_offsets), _stream())
    _check(st, "uoe_route_static")
    return r


def uoe_mlp_forward(prob: Problem, x, W1, W2, r: Routing, b1=None, b2=None, y=None, saved_h=None, ws=None,
                    check: bool = True):
    for t in (x, W1, W2, b1, b2):
        _contig(t, prob.torch_dtype)
    y = y if y is not None else torch.empty_like(x)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_MLP_FWD, x.device)
    st = _lib.uoe_mlp_forward(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2),
                              _ptr(r.expert_idx), _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.expert_offsets),
                              _ptr(y), _ptr(saved_h), _ptr(ws), ws.numel(), _stream())
    _check(st, "uoe_mlp_forward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_mlp_forward (device)")
    return y


def alloc_saved_h(prob: Problem, device="cuda") -> torch.Tensor:
    return torch.empty(uoe_max_routed_rows(prob), prob.d_e, dtype=prob.torch_dtype, device=device)


def uoe_mlp_backward(prob: Problem, x, W1, W2, W_r, r: Routing, saved_h, dy, dx=None, dW1=None, dW2=None,
                     dW_r=None, ws=None, check: bool = True):
    for t in (x, W1, W2, W_r, saved_h, dy):
        _contig(t, prob.torch_dtype)
    f32 = torch.float32
    dx = dx if dx is not None else torch.empty_like(x)
    dW1 = dW1 if dW1 is not None else torch.empty(W1.shape, dtype=f32, device=x.device)
    dW2 = dW2 if dW2 is not None else torch.empty(W2.shape, dtype=f32, device=x.device)
    dW_r = dW_r if dW_r is not None else torch.empty(W_r.shape, dtype=f32, device=x.device)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_MLP_BWD, x.device)
    st = _lib.uoe_mlp_backward(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(W1), _ptr(W2), _ptr(W_r),
                               _ptr(r.expert_idx), _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.expert_offsets),
                               _ptr(r.p_samp), _ptr(r.p_patch), _ptr(saved_h), _ptr(dy), _ptr(dx), _ptr(dW1),
                               _ptr(dW2), _ptr(dW_r), _ptr(ws), ws.numel(), _stream())
    _check(st, "uoe_mlp_backward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_mlp_backward (device)")
    return dx, dW1, dW2, dW_r


def uoe_smha_forward(prob: Problem, x, Wq, Wk, Wv, Wo, r: Routing, y=None, lse=None, ws=None, check: bool = True):
    for t in (x, Wq, Wk, Wv, Wo):
        _contig(t, prob.torch_dtype)
    y = y if y is not None else torch.empty_like(x)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_SMHA_FWD, x.device)
    st = _lib.uoe_smha_forward(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(Wq), _ptr(Wk), _ptr(Wv), _ptr(Wo),
                               _ptr(r.expert_idx), _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.expert_offsets),
                               _ptr(y), _ptr(lse), _ptr(ws), ws.numel(), _stream())
    _check(st, "uoe_smha_forward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_smha_forward (device)")
    return y


def uoe_smha_backward(prob: Problem, x, Wq, Wk, Wv, Wo, W_r, r: Routing, dy, dx=None, dWq=None, dWk=None, dWv=None,
                      dWo=None, dW_r=None, ws=None, check: bool = True):
    for t in (x, Wq, Wk, Wv, Wo, W_r, dy):
        _contig(t, prob.torch_dtype)
    f32 = torch.float32
    new = lambda like: torch.empty(like.shape, dtype=f32, device=x.device)
    dx = dx if dx is not None else torch.empty_like(x)
    dWq = dWq if dWq is not None else new(Wq)
    dWk = dWk if dWk is not None else new(Wk)
    dWv = dWv if dWv is not None else new(Wv)
    dWo = dWo if dWo is not None else new(Wo)
    dW_r = dW_r if dW_r is not None else new(W_r)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_SMHA_BWD, x.device)
    st = _lib.uoe_smha_backward(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(Wq), _ptr(Wk), _ptr(Wv), _ptr(Wo), _ptr(W_r),
                                _ptr(r.expert_idx), _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.expert_offsets),
                                _ptr(r.p_samp), _ptr(r.p_patch), _ptr(dy), _ptr(dx), _ptr(dWq), _ptr(dWk), _ptr(dWv),
                                _ptr(dWo), _ptr(dW_r), _ptr(ws), ws.numel(), _stream())
    _check(st, "uoe_smha_backward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_smha_backward (device)")
    return dx, dWq, dWk, dWv, dWo, dW_r


def uoe_route_balance(prob: Problem, p_patch, alpha: float = 1.0):
    """(lb_loss [B] float32, expert_count [B,n] int32, c_dyn [B] int32) for the patch gate written by uoe_route."""
    _contig(p_patch, torch.float32)
    dev = p_patch.device
    lb = torch.empty(prob.B, dtype=torch.float32, device=dev)
    cnt = torch.empty(prob.B, prob.n, dtype=torch.int32, device=dev)
    cd = torch.empty(prob.B, dtype=torch.int32, device=dev)
    st = _lib.uoe_route_balance(ctypes.byref(prob.c_struct()), _ptr(p_patch), ctypes.c_float(alpha), _ptr(lb), _ptr(cnt),
                                _ptr(cd), _stream())
    _check(st, "uoe_route_balance")
    return lb, cnt, cd


def uoe_route_balance_backward(prob: Problem, x, W_r, p_patch, alpha: float, dloss, ws=None, check: bool = False):
    """(dx [B,L,d], dW_r [d,n] float32): gradient of sum(dloss * lb_loss) with respect to x and W_r.

    Its kernel waits for copies with a limit; check=True synchronises and raises if a wait ran out (by default the call stays
    asynchronous and the status word of `ws`, if one is given, can be read later)."""
    _contig(x, prob.torch_dtype)
    _contig(W_r, prob.torch_dtype)
    _contig(p_patch, torch.float32)
    _contig(dloss, torch.float32)
    dx = torch.empty_like(x)
    dW_r = torch.empty(W_r.shape, dtype=torch.float32, device=x.device)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_BALANCE_BWD, x.device)
    st = _lib.uoe_route_balance_backward(ctypes.byref(prob.c_struct()), _ptr(x), _ptr(W_r), _ptr(p_patch),
                                         ctypes.c_float(alpha), _ptr(dloss), _ptr(dx), _ptr(dW_r), _ptr(ws), ws.numel(),
                                         _stream())
    _check(st, "uoe_route_balance_backward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_route_balance_backward (device)")
    return dx, dW_r


def _here(t):
    """The library works on the current device: a tensor of another one is refused."""
    dev = t.get_device()
    assert dev >= 0, "tensors must be contiguous CUDA tensors"
    if dev != torch.cuda.current_device():
        raise ValueError(f"tensors on {t.device}, but the current device is cuda:{torch.cuda.current_device()}")


_OPTIONAL = ("b1", "b2", "expert_offsets")


def _args(dev, *args):
    """Every (name, tensor, type, elements): there (or optional), contiguous, on device `dev`, of that type and size.  The library sees nothing but
    addresses, so that what this lets through is read or written in full."""
    for name, t, dtype, numel in args:
        if t is None:
            assert name in _OPTIONAL, f"{name} is missing"
        elif t.get_device() != dev or t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
            _here(t)
            raise AssertionError(f"{name}: expected {numel} contiguous elements of {dtype}, got {tuple(t.shape)} of {t.dtype}"
                                 f"{'' if t.is_contiguous() else ', not contiguous'}")


def uoe_fp8_quantize(x, layout: str, q=None, scale=None):
    """(q float8_e4m3fn, scale float32) of x [R,C] or [G,R,C] in layout "rows", "cols", "blocks" or "blocks_t" (see uoe.h)."""
    assert x.dim() in (2, 3) and x.dtype in (torch.float32, torch.bfloat16), "x must be [R,C] or [G,R,C], float32 or bfloat16"
    if layout not in FP8_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(FP8_LAYOUTS)}")
    _contig(x)
    _here(x)
    R, C = x.shape[-2:]
    blk = lambda v: -(-v // UOE_FP8_BLOCK)
    lead = tuple(x.shape[:-2])
    rows, inner = (R, C) if layout in ("rows", "blocks") else (C, R)      # of the stored matrix
    shape = (*lead, rows, blk(inner) * UOE_FP8_BLOCK)
    s_shape = (*lead, blk(inner), rows) if layout in ("rows", "cols") else (*lead, blk(rows), blk(inner))
    q = q if q is not None else torch.empty(shape, dtype=torch.float8_e4m3fn, device=x.device)
    scale = scale if scale is not None else torch.empty(s_shape, dtype=torch.float32, device=x.device)
    assert tuple(q.shape) == shape and tuple(scale.shape) == s_shape, f"expected q {shape} and scale {s_shape}"
    _args(x.get_device(), ("q", q, torch.float8_e4m3fn, q.numel()), ("scale", scale, torch.float32, scale.numel()))
    st = _lib.uoe_fp8_quantize(lead[0] if lead else 1, R, C, UOE_BF16 if x.dtype == torch.bfloat16 else UOE_F32, FP8_LAYOUTS[layout],
                               _ptr(x), _ptr(q), _ptr(scale), _stream())
    _check(st, "uoe_fp8_quantize")
    return q, scale


def uoe_fp8_transpose(x, q=None):
    """Values of 8-bit operands [.., R, C], R a multiple of 128, as [.., C, R] (see uoe.h)."""
    assert x.dim() in (2, 3), "x must be [R,C] or [G,R,C]"
    _contig(x, torch.float8_e4m3fn)
    _here(x)
    shape = (*x.shape[:-2], x.shape[-1], x.shape[-2])
    q = q if q is not None else torch.empty(shape, dtype=torch.float8_e4m3fn, device=x.device)
    assert tuple(q.shape) == shape, f"expected q {shape}"
    _args(x.get_device(), ("q", q, torch.float8_e4m3fn, q.numel()))
    st = _lib.uoe_fp8_transpose(x.shape[0] if x.dim() == 3 else 1, x.shape[-2], x.shape[-1], _ptr(x), _ptr(q), _stream())
    _check(st, "uoe_fp8_transpose")
    return q


def uoe_fp8_workspace_bytes(prob: Fp8Problem) -> int:
    return int(_lib.uoe_fp8_workspace_bytes(prob.ref))


def alloc_fp8_workspace(prob: Fp8Problem, device="cuda") -> torch.Tensor:
    nbytes = uoe_fp8_workspace_bytes(prob)
    if nbytes == 0:
        raise UoeError(1, "uoe_fp8_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        _check(_lib.uoe_workspace_init(_ptr(ws), nbytes, _stream()), "uoe_workspace_init")
    return ws


def _fp8_laid_out(t):
    """An operand whose contraction is not contiguous (the transpose of a contiguous tensor) as the products take it."""
    if t.is_contiguous() or t.dim() not in (2, 3) or not t.transpose(-1, -2).is_contiguous():
        return t
    return uoe_fp8_transpose(t.transpose(-1, -2))


def _fp8_rows(t, Kp):
    """Rows of Kp values, or all of them flat.  (A matrix that lies the other way round has the right number of elements, too.)"""
    assert t.size(-1) == Kp or t.dim() < 2, f"expected rows of {Kp} values, got {tuple(t.shape)}"


def uoe_fp8_gemm(prob: Fp8Problem, A, a_scale, W, w_scale, expert_offsets=None, C=None, ws=None, check: bool = True):
    """C [M,N] = rows A times the weights of each row's expert (8-bit operands, see uoe.h).  Without C a new tensor is returned, zero
    behind the last region.  A and W may be transposes of contiguous tensors; the call then lays their values out first."""
    n, M, N, Kb, dev, dt = prob.n, prob.M, prob.N, -(-prob.K // UOE_FP8_BLOCK), torch.cuda.current_device(), prob.torch_dtype
    Kp = Kb * UOE_FP8_BLOCK
    if C is None or ws is None:
        _here(A)
    A, W = _fp8_laid_out(A), _fp8_laid_out(W)
    if C is None:
        C = (torch.empty if expert_offsets is None else torch.zeros)(M, N, dtype=dt, device=A.device)
    ws = ws if ws is not None else alloc_fp8_workspace(prob, A.device)
    _args(dev, ("A", A, torch.float8_e4m3fn, M * Kp), ("a_scale", a_scale, torch.float32, Kb * M), ("W", W, torch.float8_e4m3fn, n * N * Kp),
          ("w_scale", w_scale, torch.float32, n * -(-N // UOE_FP8_BLOCK) * Kb), ("expert_offsets", expert_offsets, torch.int32, n + 1),
          ("C", C, dt, M * N), ("ws", ws, ws.dtype, ws.numel()))
    _fp8_rows(A, Kp)
    _fp8_rows(W, Kp)
    st = _lib.uoe_fp8_gemm(prob.ref, A.data_ptr(), a_scale.data_ptr(), W.data_ptr(), w_scale.data_ptr(), _ptr(expert_offsets), C.data_ptr(),
                           ws.data_ptr(), ws.numel(), _stream())
    _check(st, "uoe_fp8_gemm")
    if check:
        _check(uoe_read_device_status(ws), "uoe_fp8_gemm (device)")
    return C


def uoe_fp8_wgrad(prob: Fp8Problem, A, a_scale, B, b_scale, expert_offsets=None, dW=None, ws=None, check: bool = True):
    """dW [n,M,N] float32 = A B^T over the rows of each expert's region (8-bit operands, see uoe.h).  A and B may be transposes of contiguous
    tensors, as quantising by columns without turning leaves them; the call then lays their values out first."""
    n, M, N, Kb, dev = prob.n, prob.M, prob.N, -(-prob.K // UOE_FP8_BLOCK), torch.cuda.current_device()
    Kp = Kb * UOE_FP8_BLOCK
    if dW is None or ws is None:
        _here(A)
    A, B = _fp8_laid_out(A), _fp8_laid_out(B)
    dW = dW if dW is not None else torch.empty(n, M, N, dtype=torch.float32, device=A.device)
    ws = ws if ws is not None else alloc_fp8_workspace(prob, A.device)
    _args(dev, ("A", A, torch.float8_e4m3fn, M * Kp), ("a_scale", a_scale, torch.float32, Kb * M), ("B", B, torch.float8_e4m3fn, N * Kp),
          ("b_scale", b_scale, torch.float32, Kb * N), ("expert_offsets", expert_offsets, torch.int32, n + 1),
          ("dW", dW, torch.float32, n * M * N), ("ws", ws, ws.dtype, ws.numel()))
    _fp8_rows(A, Kp)
    _fp8_rows(B, Kp)
    st = _lib.uoe_fp8_wgrad(prob.ref, A.data_ptr(), a_scale.data_ptr(), B.data_ptr(), b_scale.data_ptr(), _ptr(expert_offsets), dW.data_ptr(),
                            ws.data_ptr(), ws.numel(), _stream())
    _check(st, "uoe_fp8_wgrad")
    if check:
        _check(uoe_read_device_status(ws), "uoe_fp8_wgrad (device)")
    return dW


def _weight_args(prob: Problem, W1, s1, W2, s2):
    """The two layers' weights in the problem's type, or 8-bit with their scales."""
    n, d, d_e = prob.n, prob.d, prob.d_e
    if s1 is None and s2 is None:
        return ("W1", W1, prob.torch_dtype, n * d * d_e), ("W2", W2, prob.torch_dtype, n * d_e * d)
    assert s1 is not None and s2 is not None, "8-bit weights need the scales of both layers"
    db, eb = -(-d // UOE_FP8_BLOCK), -(-d_e // UOE_FP8_BLOCK)
    return (("W1", W1, torch.float8_e4m3fn, n * d_e * db * UOE_FP8_BLOCK), ("s1", s1, torch.float32, n * eb * db),
            ("W2", W2, torch.float8_e4m3fn, n * d * eb * UOE_FP8_BLOCK), ("s2", s2, torch.float32, n * db * eb))


def _routing_args(prob: Problem, r: Routing, scores: bool):
    pairs, i32, f32 = prob.B * prob.k, torch.int32, torch.float32
    a = (("expert_idx", r.expert_idx, i32, pairs), ("patch_idx", r.patch_idx, i32, pairs * prob.c), ("gate", r.gate, f32, pairs * prob.c),
         ("routing's expert_offsets", r.expert_offsets, i32, prob.n + 1))
    if scores:
        a += (("p_samp", r.p_samp, f32, prob.B * prob.n), ("p_patch", r.p_patch, f32, prob.B * prob.n * prob.m))
    return a


def uoe_mlp_forward_fp8(prob: Problem, x, W1, s1, W2, s2, r: Routing, b1=None, b2=None, y=None, ws=None, check: bool = True):
    """uoe_mlp_forward on 8-bit weights: (W1, s1), (W2, s2) = uoe_fp8_quantize(W1 [n,d,d_e], "blocks_t"), (W2 [n,d_e,d], "blocks_t")."""
    _here(x)
    assert s1 is not None and s2 is not None, "8-bit weights need the scales of both layers"
    y = y if y is not None else torch.empty_like(x)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_MLP_FWD_FP8, x.device)
    dt, size, n = prob.torch_dtype, prob.B * prob.L * prob.d, prob.n
    _args(x.get_device(), ("x", x, dt, size), ("y", y, dt, size), ("b1", b1, dt, n * prob.d_e), ("b2", b2, dt, n * prob.d),
          ("ws", ws, ws.dtype, ws.numel()), *_weight_args(prob, W1, s1, W2, s2), *_routing_args(prob, r, False))
    _fp8_rows(W1, -(-prob.d // UOE_FP8_BLOCK) * UOE_FP8_BLOCK)
    _fp8_rows(W2, -(-prob.d_e // UOE_FP8_BLOCK) * UOE_FP8_BLOCK)
    st = _lib.uoe_mlp_forward_fp8(prob.ref, _ptr(x), _ptr(W1), _ptr(s1), _ptr(W2), _ptr(s2), _ptr(b1), _ptr(b2),
                                  _ptr(r.expert_idx), _ptr(r.patch_idx), _ptr(r.gate), _ptr(r.expert_offsets), _ptr(y), _ptr(ws),
                                  ws.numel(), _stream())
    _check(st, "uoe_mlp_forward_fp8")
    if check:
        _check(uoe_read_device_status(ws), "uoe_mlp_forward_fp8 (device)")
    return y


def uoe_mlp_tokens(prob: Problem, x, W_r, W1, W2, s1=None, s2=None, b1=None, b2=None, r: Routing | None = None, y=None, ws=None,
                   check: bool = True):
    """Router, experts and combine of a UoME layer for up to 64 tokens x [B,1,d] (or [B,d]) in two kernels; prob has L = m = c = 1.
    Weights in the problem's type, or 8-bit with their scales s1, s2 as for uoe_mlp_forward_fp8.  Fills r when given."""
    _here(x)
    y = y if y is not None else torch.empty_like(x)
    ws = ws if ws is not None else alloc_workspace(prob, UOE_OP_MLP_TOKENS, x.device)
    dt, size, n = prob.torch_dtype, prob.B * prob.L * prob.d, prob.n
    _args(x.get_device(), ("x", x, dt, size), ("y", y, dt, size), ("W_r", W_r, dt, prob.d * n), ("b1", b1, dt, n * prob.d_e), ("b2", b2, dt, n * prob.d),
          ("ws", ws, ws.dtype, ws.numel()), *_weight_args(prob, W1, s1, W2, s2), *(_routing_args(prob, r, True) if r is not None else ()))
    if s1 is not None:
        _fp8_rows(W1, -(-prob.d // UOE_FP8_BLOCK) * UOE_FP8_BLOCK)
        _fp8_rows(W2, -(-prob.d_e // UOE_FP8_BLOCK) * UOE_FP8_BLOCK)
    st = _lib.uoe_mlp_tokens(prob.ref, _ptr(x), _ptr(W_r), _ptr(W1), _ptr(s1), _ptr(W2), _ptr(s2), _ptr(b1), _ptr(b2),
                             _routing_struct(r), _ptr(y), _ptr(ws), ws.numel(), _stream())
    _check(st, "uoe_mlp_tokens")
    if check:
        _check(uoe_read_device_status(ws), "uoe_mlp_tokens (device)")
    return y


def uoe_block_workspace_bytes(att: Problem | None, mlp: Problem | None) -> int:
    pa = ctypes.byref(att.c_struct()) if att is not None else None
    pm = ctypes.byref(mlp.c_struct()) if mlp is not None else None
    return int(_lib.uoe_block_workspace_bytes(pa, pm))


def alloc_block_workspace(att: Problem | None, mlp: Problem | None, device="cuda") -> torch.Tensor:
    nbytes = uoe_block_workspace_bytes(att, mlp)
    if nbytes == 0:
        raise UoeError(1, "uoe_block_workspace_bytes")
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        _check(_lib.uoe_workspace_init(_ptr(ws), nbytes, _stream()), "uoe_workspace_init")
    return ws


def _routing_struct(r: Routing | None):
    if r is None:
        return None
    return ctypes.byref(_Routing(r.expert_idx.data_ptr(), r.patch_idx.data_ptr(), r.gate.data_ptr(), r.p_samp.data_ptr(), r.p_patch.data_ptr(),
                                 r.expert_offsets.data_ptr()))


def uoe_block_forward(att: Problem | None, mlp: Problem | None, x, weights: dict, r_att: Routing | None = None,
                      r_mlp: Routing | None = None, u=None, y=None, saved_h=None, lse=None, ws=None, check: bool = True):
    """One UoE block (SMHA half, then UoME half; either may be None) through the single C entry point.
    `weights` holds Wr_att, Wq, Wk, Wv, Wo and / or Wr_mlp, W1, W2.  Returns y (and fills u, r_att, r_mlp when given)."""
    p0 = att or mlp
    _contig(x, p0.torch_dtype)
    g = lambda name: _contig(weights.get(name), p0.torch_dtype)
    y = y if y is not None else torch.empty_like(x)
    if att is not None and mlp is not None and u is None:
        u = torch.empty_like(x)
    ws = ws if ws is not None else alloc_block_workspace(att, mlp, x.device)
    pa = ctypes.byref(att.c_struct()) if att is not None else None
    pm = ctypes.byref(mlp.c_struct()) if mlp is not None else None
    st = _lib.uoe_block_forward(pa, pm, _ptr(x), _ptr(g("Wr_att")), _ptr(g("Wq")), _ptr(g("Wk")), _ptr(g("Wv")),
                                _ptr(g("Wo")), _ptr(g("Wr_mlp")), _ptr(g("W1")), _ptr(g("W2")), _routing_struct(r_att),
                                _routing_struct(r_mlp), _ptr(u), _ptr(y), _ptr(saved_h), _ptr(lse), _ptr(ws), ws.numel(),
                                _stream())
    _check(st, "uoe_block_forward")
    if check:
        _check(uoe_read_device_status(ws), "uoe_block_forward (device)")
    return y
