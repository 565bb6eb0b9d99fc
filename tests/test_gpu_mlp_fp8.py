"""GPU parity: uoe_mlp_forward_fp8 against a plain implementation in float64, and the 8-bit operators as a training step uses them.

The rows of x are quantised alike on both sides (their quotients are exact).  The hidden values are not: the kernel's differ from the
reference's by float32 arithmetic, da (K 2^-23 sum |terms|, phi's growth 1.13 and its 2^-20), and where a rounding border to e4m3, or a
scale's border, lies within da of the value, either neighbour is right.  The reference therefore takes the quantised values at both ends
(with either scale), and what lies between them times |W2| enters the bound; everything else is float32 sums, the bfloat16 rounding of the
experts' outputs (half a step, 2^-8) and of the result.
"""
import pytest
import torch

import uoe_inputs as gen
from tests.helpers import problem_of, to_dev, to_f64
from tests.test_gpu_fp8 import BLOCK, _e4m3_nearest, _quantize_ref
from tests.test_gpu_mlp_tokens import _phi

pytestmark = pytest.mark.gpu


def _w(**kw):
    base = dict(dtype="bf16", w_std=0.08, H=0, d_h=0)
    base.update(kw)
    return gen.tiny(**base)


CASES = {
    "small": (_w(d=64, d_ff=4 * 64), {}),
    "odd_widths": (_w(B=5, L=112, L_valid=100, m=7, c=4, d=136, n=3, k=2, d_ff=3 * 72), dict(bias=True)),
    "patches_of_24": (_w(B=4, L=240, L_valid=230, m=10, c=4, d=200, n=5, k=3, d_ff=5 * 264, act="gelu_erf"), dict(gate=False)),
    "one_token_patches": (_w(B=3, L=40, L_valid=37, m=40, c=9, d=72, n=4, k=2, d_ff=4 * 40, act="gelu_tanh"), dict(bias=True, residual=False)),
    "one_sample_one_expert": (_w(B=1, L=8, L_valid=5, m=1, c=1, d=8, n=1, k=1, d_ff=8), {}),
    "unused_slots": (_w(B=3, L=128, L_valid=20, m=8, c=6, d=256, n=4, k=2, d_ff=4 * 128), {}),
    "several_tiles": (_w(B=6, L=512, L_valid=500, m=16, c=8, d=384, n=6, k=3, d_ff=6 * 256, w_std=0.05), {}),
    "any_scale": (_w(B=3, L=96, L_valid=96, m=6, c=3, d=192, n=4, k=2, d_ff=4 * 136), dict(any_scale=True)),
    "pairs_of_ctas": (_w(B=40, L=1152, L_valid=1152, m=9, c=3, d=256, n=4, k=2, d_ff=4 * 320, w_std=0.05), {}),
    "gathered_patches_of_8": (_w(B=14, L=1152, L_valid=1130, m=144, c=48, d=200, n=8, k=4, d_ff=8 * 320, w_std=0.05), dict(bias=True)),
    "gathered_patches_of_64": (_w(B=9, L=2048, L_valid=2048, m=32, c=9, d=264, n=12, k=4, d_ff=12 * 392, act="gelu_erf", w_std=0.05), {}),
    "hidden_width_of_33": (_w(B=3, L=64, L_valid=64, m=4, c=3, d=72, n=4, k=2, d_ff=4 * 33, act="gelu_tanh"), dict(bias=True)),
    "by_patch": (_w(B=11, L=1280, L_valid=1201, m=10, c=5, d=520, n=7, k=5, d_ff=7 * 200, act="gelu_tanh", w_std=0.05), dict(bias=True)),
    "by_patch_one_block": (_w(B=30, L=768, L_valid=768, m=6, c=2, d=264, n=5, k=2, d_ff=5 * 40), dict(gate=False, residual=False)),
    "by_patch_all_experts": (_w(B=20, L=1024, L_valid=900, m=8, c=8, d=136, n=3, k=3, d_ff=3 * 392, w_std=0.05), {}),
    "gathered_whole_samples": (_w(B=7, L=256, L_valid=256, m=2, c=2, d=136, n=8, k=2, d_ff=8 * 136), {}),
}


def _row_values(rows):
    q, s = _quantize_ref(rows, 1)
    return (q * s.repeat_interleave(BLOCK, 1))[:, :rows.shape[1]]


def _between(a, da):
    """(quantised values of a, how far apart the quantised ends of a +- da can be), a scale per row and 128 columns."""
    R, C = a.shape
    Cb = -(-C // BLOCK)
    pad = lambda v: torch.nn.functional.pad(v, (0, Cb * BLOCK - C)).view(R, Cb, BLOCK)
    a, da = pad(a), pad(da)
    scale = lambda top: torch.exp2(torch.ceil(torch.log2(top.clamp(min=2.0 ** -100) / 448) - 1e-13))
    s0, s1, mid = (scale(v)[..., None] for v in ((a.abs() - da).amax(2), (a.abs() + da).amax(2), a.abs().amax(2)))
    e4 = lambda v, s: _e4m3_nearest((v / s).clamp(-448, 448)) * s
    ends = torch.stack([e4(a - da, s0), e4(a + da, s0), e4(a - da, s1), e4(a + da, s1), e4(a, mid)])
    flat = lambda v: v.reshape(R, -1)[:, :C]
    return flat(ends[4]), flat(ends.amax(0) - ends.amin(0))


def _weights(uoe, W, any_scale, seed):
    q, s = uoe.uoe_fp8_quantize(to_dev(W), "blocks_t")
    if any_scale:
        s *= (0.5 + torch.rand(s.shape, generator=torch.Generator().manual_seed(seed))).cuda()
    K = W.f64.shape[1]
    v = (q.float().cpu().double() * s.cpu().double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]].repeat_interleave(BLOCK, 2))[..., :K]
    return q, s, v.transpose(1, 2)


def _setup(name):
    import paper_2503_02495_b200 as uoe
    w, o = CASES[name]
    prob = problem_of(w, "mlp", residual=o.get("residual", True), gate=o.get("gate", True), fp8_any_scale=o.get("any_scale", False))
    x, Wr = gen.make_x(w), gen.store(gen.make_router(w).f64 * 20, w.dtype)
    W1, W2 = gen.make_mlp_weights(w)
    b = [gen.store(gen.normal(w.seed, 20 + i, shape, 0.3), "bf16") if o.get("bias") else None for i, shape in enumerate([(w.n, w.d_e), (w.n, w.d)])]
    r = uoe.uoe_route(prob, to_dev(x), to_dev(Wr))
    q1, q2 = _weights(uoe, W1, prob.fp8_any_scale, 1), _weights(uoe, W2, prob.fp8_any_scale, 2)
    return w, prob, x, r, q1, q2, b


def _reference(w, prob, x, r, v1, v2, b):
    X = torch.from_numpy(x.f64).view(-1, w.d)
    y, err = (X.clone() if prob.residual else torch.zeros_like(X)), torch.zeros_like(X)
    e, pj, gate = r.expert_idx.cpu(), r.patch_idx.cpu(), r.gate.cpu().double()
    b1, b2 = (None if q is None else torch.from_numpy(q.f64) for q in b)
    for i in range(w.n):
        rows, wt = [], []
        for s_, k_ in (e == i).nonzero().tolist():
            for u, j in enumerate(pj[s_, k_].tolist()):
                if j < 0:
                    continue
                for t in range(j * w.l_p, min((j + 1) * w.l_p, w.L_valid)):
                    rows.append(s_ * w.L + t)
                    wt.append(gate[s_, k_, u] if prob.gate else 1.0)
        if not rows:
            continue
        rows, wt = torch.tensor(rows), torch.tensor(wt, dtype=torch.float64)[:, None]
        xq = _row_values(X[rows])
        h = xq @ v1[i] + (0 if b1 is None else b1[i])
        dh = (4 * w.d + 600) * 2.0 ** -23 * (xq.abs() @ v1[i].abs())       # (blocks are padded to 128)
        a = _phi(h, w.act)
        aq, gap = _between(a, 1.13 * dh + 2.0 ** -20 * a.abs() + 1e-30)
        z = aq @ v2[i] + (0 if b2 is None else b2[i])
        dz = gap @ v2[i].abs() + (4 * w.d_e + 600) * 2.0 ** -23 * (aq.abs() @ v2[i].abs())
        dz = dz + 2.0 ** -8 * (z.abs() + dz)
        y.index_add_(0, rows, wt * z)
        err.index_add_(0, rows, wt * (dz + 2.0 ** -21 * z.abs()))
    return y, err + 2.0 ** -8 * (y.abs() + err) + 1e-30


@pytest.mark.parametrize("name", list(CASES))
def test_mlp_fp8(name):
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, v1), (W2, s2, v2), b = _setup(name)
    bd = [None if q is None else to_dev(q) for q in b]
    got = uoe.uoe_mlp_forward_fp8(prob, to_dev(x), W1, s1, W2, s2, r, b1=bd[0], b2=bd[1])
    y, bound = _reference(w, prob, x, r, v1, v2, b)
    diff = (torch.from_numpy(to_f64(got)).view(y.shape) - y).abs()
    pad = torch.arange(w.L).repeat(w.B) >= w.L_valid
    assert (diff[~pad] <= bound[~pad]).all(), float((diff / bound)[~pad].max())
    assert torch.equal(got.view(-1, w.d)[pad.cuda()], to_dev(x).view(-1, w.d)[pad.cuda()] * (1 if prob.residual else 0))
    assert torch.equal(got, uoe.uoe_mlp_forward_fp8(prob, to_dev(x), W1, s1, W2, s2, r, b1=bd[0], b2=bd[1]))


@pytest.mark.parametrize("name", ["several_tiles", "gathered_patches_of_8", "small", "by_patch"])
def test_captured_and_on_two_streams(name):
    """Replays follow the tensors' contents; two streams with a workspace each do not meet."""
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, v1), (W2, s2, v2), b = _setup(name)
    xd = to_dev(x)
    x2 = xd.flip(0).contiguous()
    r2 = type(r)(**{k: v.clone() if torch.is_tensor(v) else v for k, v in vars(uoe.uoe_route(prob, x2, to_dev(gen.store(gen.make_router(w).f64 * 20, w.dtype)))).items()})
    run = lambda xx, rr, ws: uoe.uoe_mlp_forward_fp8(prob, xx, W1, s1, W2, s2, rr, ws=ws, check=False)      # (the check waits for the device)
    ws = [uoe.alloc_workspace(prob, uoe.UOE_OP_MLP_FWD_FP8) for _ in range(2)]
    want, want2 = run(xd, r, ws[0]).clone(), run(x2, r2, ws[0]).clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i, (xx, rr) in enumerate(((xd, r), (x2, r2))):
            with torch.cuda.stream(streams[i]):
                got[i] = run(xx, rr, ws[i])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want2)
    held = xd.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(held, r, ws[0])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    held.copy_(x2)
    for a, c in ((r.expert_idx, r2.expert_idx), (r.patch_idx, r2.patch_idx), (r.gate, r2.gate), (r.expert_offsets, r2.expert_offsets)):
        a.copy_(c)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want2)


def test_prompt_then_tokens():
    """Serving: a prompt through the routed layer, then tokens one by one through the few-token kernels, on the same 8-bit weights."""
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, v1), (W2, s2, v2), b = _setup("small")
    y = uoe.uoe_mlp_forward_fp8(prob, to_dev(x), W1, s1, W2, s2, r)
    one = problem_of(w, "mlp", B=1, L=1, L_valid=1, m=1, c=1)
    Wr = to_dev(gen.store(gen.make_router(w).f64 * 20, w.dtype))
    ws = uoe.alloc_workspace(one, uoe.UOE_OP_MLP_TOKENS)
    h = y[0, w.L_valid - 1].view(1, 1, w.d).contiguous()
    for _ in range(4):
        h2 = uoe.uoe_mlp_tokens(one, h, Wr, W1, W2, s1=s1, s2=s2, ws=ws)
        rt = uoe.uoe_route(one, h, Wr)
        X = h.cpu().double().view(-1)
        ref = X.clone()
        for i, g in zip(rt.expert_idx[0].tolist(), rt.gate.flatten().tolist()):
            ref += g * (_phi(X @ v1[i], w.act) @ v2[i])
        assert (h2.cpu().double().view(-1) - ref).abs().max() <= 2e-2 * ref.abs().max()
        h = h2


def test_training_step_of_an_expert_layer():
    """Forward product, gradient of the rows (weights quantised the other way round) and of the weights, against float64 on the quantised
    operands, and the formula against differences: <dy, C(x + t v) - C(x)> = t <dx, v> and the same for W, exactly (C is bilinear)."""
    import paper_2503_02495_b200 as uoe
    g = torch.Generator().manual_seed(5)
    n, K, N, off = 3, 200, 136, [0, 256, 256, 640]
    live = torch.zeros(640, 1)
    live[:200], live[256:600] = 1, 1
    x, dy = torch.randn(640, K, generator=g) * live, torch.randn(640, N, generator=g) * live
    W = torch.randn(n, K, N, generator=g) * K ** -0.5
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    q = lambda t, lay: uoe.uoe_fp8_quantize(t.cuda(), lay)
    vec = lambda qs: qs[0].float().cpu().double() * qs[1].cpu().double().t().repeat_interleave(BLOCK, 1)
    blk = lambda qs: qs[0].float().cpu().double() * qs[1].cpu().double().repeat_interleave(BLOCK, 1)[:, :qs[0].shape[1]].repeat_interleave(BLOCK, 2)
    xr, Wt = q(x, "rows"), q(W, "blocks_t")                       # W^T: [n, N, K]
    C = uoe.uoe_fp8_gemm(uoe.Fp8Problem(n, 640, N, K, "f32"), *xr, *Wt, o)
    dr, Wb = q(dy, "rows"), q(W, "blocks")                        # [n, K, N]: contracted over N
    dx = uoe.uoe_fp8_gemm(uoe.Fp8Problem(n, 640, K, N, "f32"), *dr, *Wb, o)
    xc, dc = q(x, "cols"), q(dy, "cols")
    dW = uoe.uoe_fp8_wgrad(uoe.Fp8Problem(n, K, N, 640, "f32"), *xc, *dc, o)
    assert torch.equal(blk(Wt).transpose(1, 2)[:, :K], blk(Wb)[..., :N])      # one set of values whichever way they are stored
    for e in range(n):
        s = slice(off[e], off[e + 1])
        w = blk(Wb)[e][:, :N]
        for got, a, b in ((C[s], vec(xr)[s, :K], w), (dx[s], vec(dr)[s, :N], w.t()), (dW[e], vec(xc)[:, s], vec(dc)[:, s].t())):
            tol = (4 * max(K, N, 640) + 16) * 2.0 ** -23 * (a.abs() @ b.abs()) + 1e-30
            assert ((got.cpu().double() - a @ b).abs() <= tol).all()
    # against differences of the unquantised product: what remains is the operands' rounding, at most 2^-4 of each factor
    v = torch.randn(640, K, generator=g).double() * live
    for e in range(n):
        s = slice(off[e], off[e + 1])
        diff = ((dy[s].double() @ W[e].double().t()) * v[s]).sum()
        room = (2 * 2.0 ** -4 + 2.0 ** -8) * ((dy[s].double().abs() @ W[e].double().abs().t()) * v[s].abs()).sum()
        assert (dx[s].cpu().double() * v[s]).sum().sub(diff).abs() <= room
