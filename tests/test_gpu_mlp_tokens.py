"""GPU parity: uoe_mlp_tokens (router, experts and combine for a few tokens) against a plain implementation in float64.

Bounds, element by element, from the float64 values themselves.  With u = 2^-24 (float32) and K terms a float32 sum is off by at most
K 2^-23 sum |terms| (any order of additions).  Router: a score off by ds changes a softmax gate by at most a factor exp(2 ds), the
combine weight (its square) by twice that; expf and the division add 2^-20.  Hidden rows: phi grows no faster than 1.13; it is evaluated to
2^-20 of its value and stored with half a step (2^-8 for bfloat16, 2^-24 for float32).  The result's own rounding is half a step again.
8-bit weights: the rows' two e4m3 terms s (hi + lo / 16), s <= max / 224, are exact from 2^-6 s on; below, 16 times what hi leaves is rounded
to steps of 2^-9, half a step 2^-10 / 16 s = 2^-14 s < 2^-21 max, max the largest magnitude in the block of 128.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BLOCK = 128


def _phi(h, act):
    if act == "silu":
        return h * torch.sigmoid(h)
    if act == "identity":
        return h
    return torch.nn.functional.gelu(h, approximate="none" if act == "gelu_erf" else "tanh")


def _case(T, d, d_e, n, k, weights="bf16", act="silu", bias=False, gate=True, residual=True, seed=0, spread=0):
    return dict(spread=spread, T=T, d=d, d_e=d_e, n=n, k=k, weights=weights, act=act, bias=bias, gate=gate, residual=residual, seed=seed)


CASES = {
    "one": _case(1, 64, 32, 2, 1),
    "smallest": _case(1, 8, 8, 1, 1),
    "one_of_many": _case(1, 512, 256, 8, 4),
    "odd": _case(5, 136, 72, 5, 3, bias=True, act="gelu_erf"),
    "odd_tail": _case(3, 200, 104, 7, 2, bias=True, act="gelu_tanh", residual=False),
    "sixteen": _case(16, 256, 136, 6, 3, gate=False),
    "seventeen": _case(17, 264, 136, 6, 3, bias=True),
    "thirty_two_experts": _case(32, 128, 64, 32, 8),
    "thirty_three": _case(33, 128, 80, 9, 2, bias=True),
    "sixty_four": _case(64, 320, 64, 4, 4),
    "all_experts": _case(7, 96, 48, 3, 3, act="identity"),
    "wide": _case(2, 2056, 1032, 4, 2),
    "fp8_one": _case(1, 64, 32, 2, 1, "fp8"),
    "fp8_smallest": _case(1, 8, 8, 1, 1, "fp8"),
    "fp8_odd": _case(5, 136, 72, 5, 3, "fp8", bias=True, act="gelu_erf"),
    "fp8_tail": _case(18, 328, 200, 7, 2, "fp8", residual=False),
    "fp8_many": _case(64, 264, 136, 6, 3, "fp8", bias=True, gate=False),
    "fp8_wide": _case(4, 2056, 1032, 4, 2, "fp8"),
    "fp8_range": _case(6, 392, 200, 5, 2, "fp8", act="identity", residual=False, spread=24),
    "f32_one": _case(1, 64, 32, 2, 1, "f32"),
    "f32_smallest": _case(1, 4, 4, 1, 1, "f32"),
    "f32_odd": _case(9, 132, 68, 5, 3, "f32", bias=True, act="gelu_erf"),
    "f32_many": _case(50, 260, 100, 12, 4, "f32", act="gelu_tanh", gate=False),
}


def make(c):
    dt = torch.float32 if c["weights"] == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(100 + c["seed"])
    rn = lambda *s, std=1.0: (torch.randn(*s, generator=g, dtype=torch.float64) * std).to(dt)
    n, d, d_e = c["n"], c["d"], c["d_e"]
    x = rn(c["T"], 1, d)
    if c["spread"]:       # values of very different sizes in a row, and so hidden values too; the router hardly sees the small ones
        x = (x.double() * torch.exp2(-torch.randint(0, c["spread"], (1, 1, d), generator=g).double())).to(dt)
    return dict(x=x, Wr=rn(d, n, std=3 * d ** -0.5), W1=rn(n, d, d_e, std=d ** -0.5), W2=rn(n, d_e, d, std=d_e ** -0.5),
                b1=rn(n, d_e, std=0.3) if c["bias"] else None, b2=rn(n, d, std=0.3) if c["bias"] else None)


def _terms_error(v):
    """Per element of v [K]: 2^-21 of the largest in its block of 128, where the element is not exact for certain."""
    K = v.shape[0]
    top = torch.nn.functional.pad(v.abs(), (0, -K % BLOCK)).view(-1, BLOCK).amax(1).repeat_interleave(BLOCK)[:K]
    return torch.where(v.abs() < 2.0 ** -5 / 224 * top, 2.0 ** -21 * top, torch.zeros_like(top))


def reference(c, x, Wr, W1, W2, b1, b2, experts=None):
    """(y, bound on a float32 / bfloat16 implementation's error, experts [T,k], p [T,n]) in float64; W1 [n,d,d_e], W2 [n,d_e,d] values."""
    half = 2.0 ** -24 if c["weights"] == "f32" else 2.0 ** -8
    d, d_e, k = c["d"], c["d_e"], c["k"]
    x = x.double().view(-1, d)
    s = x @ Wr.double()
    ds = (d + 8) * 2.0 ** -23 * (x.abs() @ Wr.double().abs())
    p = torch.softmax(s, 1)
    e = p.sort(dim=1, descending=True, stable=True).indices[:, :k].sort(1).values
    top = p.sort(dim=1, descending=True).values
    if k < c["n"]:        # the choice itself is not in question
        assert ((top[:, k - 1] - top[:, k]) / top[:, k - 1]).min() > 1e-4
    y, err = (x.clone() if c["residual"] else torch.zeros_like(x)), torch.zeros_like(x)
    rel_p = 2 * ds.amax(1, keepdim=True) + 2.0 ** -20
    for t in range(x.shape[0]):
        for i in e[t].tolist():
            h, hb = x[t] @ W1[i].double(), (d + 8) * 2.0 ** -23 * (x[t].abs() @ W1[i].double().abs())
            if c["weights"] == "fp8":
                hb = hb + _terms_error(x[t]) @ W1[i].double().abs()
            if b1 is not None:
                h = h + b1[i].double()
            a = _phi(h, c["act"])
            da = 1.13 * hb + (2.0 ** -20 + half) * a.abs() + 2.0 ** -126
            z = a @ W2[i].double() + (b2[i].double() if b2 is not None else 0)
            dz = da @ W2[i].double().abs() + (d_e * k + 16) * 2.0 ** -23 * (a.abs() @ W2[i].double().abs()) + 2.0 ** -22 * z.abs()
            if c["weights"] == "fp8":
                dz = dz + _terms_error(a) @ W2[i].double().abs()
            w = p[t, i] ** 2 if c["gate"] else torch.tensor(1.0, dtype=torch.float64)
            y[t] += w * z
            err[t] += w * dz + (w * 2 * rel_p[t] * z.abs() if c["gate"] else 0) + k * 2.0 ** -23 * (w * z).abs()
    return y, err + half * (y.abs() + err) + 2.0 ** -23 * x.abs(), e, p


def run(c, m, **kw):
    import paper_2503_02495_b200 as uoe
    prob = uoe.Problem(B=c["T"], L=1, L_valid=1, d=c["d"], n=c["n"], k=c["k"], m=1, c=1, d_e=c["d_e"], act=c["act"], gate=c["gate"],
                       residual=c["residual"], dtype="f32" if c["weights"] == "f32" else "bf16")
    dev = {q: v.cuda() if v is not None else None for q, v in m.items()}
    s1 = s2 = None
    W1, W2 = dev["W1"], dev["W2"]
    v1, v2 = m["W1"], m["W2"]
    if c["weights"] == "fp8":
        W1, s1 = uoe.uoe_fp8_quantize(W1, "blocks_t")
        W2, s2 = uoe.uoe_fp8_quantize(W2, "blocks_t")
        g = torch.Generator().manual_seed(7)
        s1 *= (0.5 + torch.rand(s1.shape, generator=g)).cuda()         # any scales
        s2 *= (0.5 + torch.rand(s2.shape, generator=g)).cuda()
        val = lambda q, s, K: (q.float().cpu().double() * s.cpu().double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
                               .repeat_interleave(BLOCK, 2))[..., :K].transpose(1, 2)
        v1, v2 = val(W1, s1, c["d"]), val(W2, s2, c["d_e"])
    call = lambda **q: uoe.uoe_mlp_tokens(prob, dev["x"], dev["Wr"], W1, W2, s1=s1, s2=s2, b1=dev["b1"], b2=dev["b2"], **q)
    return prob, call, v1, v2


def _check(got, y, bound):
    diff = (got.double().cpu().view(y.shape) - y).abs()
    assert (diff <= bound).all(), float((diff / bound).max())


@pytest.mark.parametrize("name", list(CASES))
def test_tokens(name):
    import paper_2503_02495_b200 as uoe
    c = CASES[name]
    m = make(c)
    prob, call, v1, v2 = run(c, m)
    r = uoe.alloc_routing(prob)
    got = call(r=r)
    y, bound, e, p = reference(c, m["x"], m["Wr"], v1, v2, m["b1"], m["b2"])
    assert torch.equal(r.expert_idx.cpu().long(), e)
    _check(got, y, bound)
    assert (r.p_samp.cpu().double() - p).abs().max() <= 1e-4 and torch.equal(r.p_samp, r.p_patch.view_as(r.p_samp))
    assert (r.patch_idx == 0).all()
    sel = torch.gather(r.p_samp, 1, r.expert_idx.long())
    assert torch.equal(r.gate.view_as(sel), sel * sel if c["gate"] else torch.ones_like(sel))
    cnt = torch.bincount(e.flatten(), minlength=c["n"])
    assert r.expert_offsets.cpu().tolist() == [0] + torch.cumsum((cnt + 127) // 128 * 128, 0).tolist()
    assert torch.equal(got, call())                   # the same bits each time, with or without the routing arrays


def test_tokens_equal_the_general_layer():
    """The same layer through uoe_route and uoe_mlp_forward (128-row tiles), routing included."""
    import paper_2503_02495_b200 as uoe
    c = _case(24, 512, 256, 8, 4)
    m = make(c)
    prob, call, _, _ = run(c, m)
    r = uoe.alloc_routing(prob)
    got = call(r=r)
    x = m["x"].cuda()
    r2 = uoe.uoe_route(prob, x, m["Wr"].cuda())
    for f in ("expert_idx", "patch_idx", "expert_offsets"):
        assert torch.equal(getattr(r, f), getattr(r2, f)), f
    y2 = uoe.uoe_mlp_forward(prob, x, m["W1"].cuda(), m["W2"].cuda(), r2)
    y, bound, _, _ = reference(c, m["x"], m["Wr"], m["W1"], m["W2"], None, None)
    _check(got, y, bound)
    assert (got.double() - y2.double()).abs().max() <= 2e-2 * y.abs().max()


@pytest.mark.parametrize("weights", ["bf16", "fp8", "f32"])
def test_an_expert_nobody_chose_may_hold_anything(weights):
    """Weights of experts without a token are not looked at, and an expert's infinities stay with the tokens that chose it."""
    import paper_2503_02495_b200 as uoe
    c = _case(6, 64, 32, 4, 1, "bf16" if weights == "fp8" else weights, gate=False)
    m = make(c)
    prob, call, _, _ = run(c, m)
    r = uoe.alloc_routing(prob)
    ref = call(r=r)
    used = sorted(set(r.expert_idx.flatten().tolist()))
    for bad in range(4):
        m2 = {q: v.clone() if v is not None else None for q, v in m.items()}
        m2["W2"][bad] = float("inf")
        m2["W1"][bad, 0, 0] = float("nan")
        got = run(c, m2)[1]()
        keep = (r.expert_idx.flatten() != bad)
        assert torch.equal(got[keep], ref[keep])
        assert bad not in used or not torch.isfinite(got[~keep]).all()


def test_a_token_with_a_nan_spoils_only_itself():
    import paper_2503_02495_b200 as uoe
    c = _case(20, 128, 64, 6, 2)
    m = make(c)
    prob, call, _, _ = run(c, m)
    ref = call()
    m["x"][11, 0, 5] = float("nan")
    r = uoe.alloc_routing(prob)
    got = run(c, m)[1](r=r)
    keep = torch.arange(20) != 11
    assert torch.equal(got[keep], ref[keep]) and torch.isnan(got[11]).all()
    assert r.expert_idx[11].tolist() == [0, 1]


def test_tokens_in_a_graph_and_on_other_streams():
    """A captured call replayed on new inputs; two streams with a workspace each; what lies behind y stays as it was."""
    import paper_2503_02495_b200 as uoe
    c = _case(3, 256, 128, 6, 2, "fp8")
    m = make(c)
    prob, call, _, _ = run(c, m)
    x = m["x"].cuda()
    W1, s1 = uoe.uoe_fp8_quantize(m["W1"].cuda(), "blocks_t")
    W2, s2 = uoe.uoe_fp8_quantize(m["W2"].cuda(), "blocks_t")
    Wr = m["Wr"].cuda()
    f = lambda x, y, ws: uoe.uoe_mlp_tokens(prob, x, Wr, W1, W2, s1=s1, s2=s2, y=y, ws=ws, check=False)
    buf = torch.full((5, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = uoe.alloc_workspace(prob, uoe.UOE_OP_MLP_TOKENS)
    xs = [x, x.flip(0).contiguous(), -x]
    refs = [f(v, torch.empty_like(v), ws).clone() for v in xs]
    torch.cuda.synchronize()
    xin, y = x.clone(), buf[:3].view(3, 1, 256)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(xin, y, ws)
    for v, r in zip(xs, refs):
        xin.copy_(v)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, r) and (buf[3:] == 7).all()
    st = [torch.cuda.Stream() for _ in range(2)]
    outs, wss = [torch.empty_like(x) for _ in st], [uoe.alloc_workspace(prob, uoe.UOE_OP_MLP_TOKENS) for _ in st]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, s in enumerate(st):
            with torch.cuda.stream(s):
                f(xs[q], outs[q], wss[q])
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for o, r in zip(outs, refs))
    assert uoe.uoe_read_device_status(ws) == 0
