"""The operators around 8-bit expert weights and the layer for a few tokens: what programs have them do, and their plain form.

A case is a plain dict; `op` says which operator it is:
  quantize   uoe_fp8_quantize: float -> 8-bit floating point (e4m3) with a scale for each block
  gemm       uoe_fp8_gemm: rows (a scale per row and 128 columns) times expert weights (a scale per 128 x 128 block)
  wgrad      uoe_fp8_wgrad: gradient of expert weights from two operands with a scale per 128 routed rows
  mlp        uoe_mlp_forward_fp8: the routed MLP layer on 8-bit weights
  tokens     uoe_mlp_tokens: router, experts and combine for a few tokens

`own` false: elementary torch operations; true: the calls a program makes of the library.  listed() holds the cases, draw()
makes more of the same ranges, prepare() what a program has in hand before the call, run() is one pass, work() what it cannot do
without, exact() the operator's definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
F8 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ceil(a, b):
    return -(-a // b)


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------

def listed():
    lm = dict(d=512, n=8, k=4, d_e=256)                 # the causal language-model block
    scale = dict(d=4096, n=16, k=4, d_e=1024)           # the large MLP block
    return [
        # activations of four sequences of the large block on their way into a product
        dict(name="quantize_activations", op="quantize", layout="rows", G=1, R=16384, C=4096, dtype="bf16"),
        # first-layer weights of the large block, laid out once before serving (each step in training)
        dict(name="quantize_weights", op="quantize", layout="blocks_t", G=16, R=4096, C=1024, dtype="bf16"),
        # one token against a square projection: latency and weight bandwidth
        dict(name="gemm_one_token", op="gemm", n=1, rows=1, skew=0.0, slack=0, N=4096, K=4096, out="bf16"),
        # first layer of the language-model block: many experts, short contraction, ragged regions
        dict(name="gemm_lm_experts", op="gemm", n=8, rows=16384, skew=0.7, slack=1024, N=256, K=512, out="bf16"),
        # first layer of the large block
        dict(name="gemm_scale_experts", op="gemm", n=16, rows=32768, skew=0.3, slack=2048, N=1024, K=4096, out="bf16"),
        # sizes that no tile divides, float32 out
        dict(name="gemm_odd", op="gemm", n=3, rows=1334, skew=2.0, slack=77, N=333, K=1000, out="f32"),
        # weight gradients of the two blocks above
        dict(name="wgrad_lm", op="wgrad", n=8, rows=16384, skew=0.7, M=512, N=256),
        dict(name="wgrad_scale", op="wgrad", n=16, rows=32768, skew=0.3, M=4096, N=1024),
        # the layers themselves: serving a batch of prompts
        dict(name="mlp_lm", op="mlp", B=16, L_valid=512, l_p=32, m=16, c=8, act="silu", bias=False, gate=True, **lm),
        dict(name="mlp_scale", op="mlp", B=4, L_valid=4096, l_p=128, m=32, c=16, act="silu", bias=False, gate=True, **scale),
        # decoding: one token of the language-model block, eight of the large one on 8-bit weights
        dict(name="tokens_lm_one", op="tokens", T=1, weights="bf16", act="silu", bias=False, gate=True, **lm),
        dict(name="tokens_scale_eight", op="tokens", T=8, weights="fp8", act="silu", bias=False, gate=True, **scale),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "gemm", "wgrad", "mlp", "tokens", "tokens"])
    if op == "quantize":
        layout, G = rng.choice(["rows", "cols", "blocks", "blocks_t"]), rng.choice([1, 1, _log(rng, 1, 16)])
        C = _log(rng, 1, 8192)
        R = _log(rng, 1, max(1, min(30000, (1 << 26) // (C * G))))
        return dict(op=op, layout=layout, G=G, R=R, C=C, dtype=rng.choice(["bf16", "f32"]))
    if op in ("gemm", "wgrad"):
        n = rng.choice([1, 1, _log(rng, 1, 16)]) if op == "gemm" else _log(rng, 1, 16)
        rows, skew = _log(rng, 1, 30000), rng.choice([0.0, 0.5, 1.0, 3.0])
        if op == "wgrad":
            return dict(op=op, n=n, rows=rows, skew=skew, M=_log(rng, 8, 4096), N=_log(rng, 8, 1024))
        return dict(op=op, n=n, rows=rows, skew=skew, slack=rng.choice([0, rng.randrange(1, 500)]), N=_log(rng, 8, 2048), K=_log(rng, 16, 4096),
                    out=rng.choice(["bf16", "bf16", "f32"]))
    n = _log(rng, 2, 16)
    k = rng.randrange(1, min(n, 8) + 1)
    base = dict(d=8 * _log(rng, 8, 256), n=n, k=k, d_e=8 * _log(rng, 4, 128), act=rng.choice(["silu", "gelu_erf", "gelu_tanh"]),
                bias=rng.random() < 0.3, gate=rng.random() < 0.7)
    if op == "tokens":
        return dict(op=op, T=_log(rng, 1, 64), weights=rng.choice(["bf16", "bf16", "fp8", "fp8", "f32"]), **base)
    l_p, m = rng.choice([1, 8, 16, 24, 32, 64, 128]), _log(rng, 2, 32)
    c, B = rng.randrange(1, m + 1), _log(rng, 1, 16)
    k = base["k"] = min(k, 4)
    while B * k * c * l_p > 32768 and B > 1:
        B //= 2
    return dict(op=op, B=B, L_valid=m * l_p - rng.randrange(0, l_p), l_p=l_p, m=m, c=c, **base)


# ---------------------------------------------------------------------------------------------------------------------
# what a program holds
# ---------------------------------------------------------------------------------------------------------------------

def _counts(case):
    """Rows of every expert: shares that fall off as (place + 1) ** -skew, the places in a fixed order that mixes large and small;
    what rounding leaves over goes to the first place.  A strong skew leaves experts without rows."""
    n, rows = case["n"], case["rows"]
    share = [(i + 1) ** -case["skew"] for i in range(n)]
    cnt = [int(rows * s / sum(share)) for s in share]
    cnt[0] += rows - sum(cnt)
    order = sorted(range(n), key=lambda i: (i * 7 + 3) % n if n % 7 else (i * 5 + 3) % n)
    return [cnt[i] for i in order]


def _regions(rows):
    """Expert regions: every expert's rows, each region padded to a multiple of 128."""
    off = [0]
    for r in rows:
        off.append(off[-1] + _ceil(r, BLOCK) * BLOCK)
    return off


def _amax_scale(amax):
    """(1 / s, s): s the smallest power of two with amax <= 448 s (amax at least 2^-100), so that x / s is exact."""
    f, e = torch.frexp(amax.clamp_min(2.0 ** -100))
    e = e - 9 + (f > 0.875)
    one = torch.ones_like(f)
    return torch.ldexp(one, -e), torch.ldexp(one, e)


def _q_vec(x):
    """x [..., R, C] -> q [..., R, C padded to 128] e4m3 and scale [..., C / 128, R]: a scale per row and 128 columns."""
    x = x.float()
    C = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -C % BLOCK))
    t = x.unflatten(-1, (-1, BLOCK))
    r, s = _amax_scale(t.abs().amax(-1))
    return (t * r.unsqueeze(-1)).flatten(-2).to(F8), s.transpose(-1, -2).contiguous()


def _q_blk(x):
    """x [..., R, C] -> q [..., R, C padded] e4m3 and scale [..., R / 128, C / 128]: a scale per 128 x 128 block."""
    x = x.float()
    R, C = x.shape[-2:]
    x = torch.nn.functional.pad(x, (0, -C % BLOCK, 0, -R % BLOCK))
    t = x.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, BLOCK))            # [..., Rb, 128, Cb, 128]
    r, s = _amax_scale(t.abs().amax((-3, -1)))
    q = (t * r.unsqueeze(-1).unsqueeze(-3)).to(F8)
    return q.flatten(-2).flatten(-3, -2)[..., :R, :].contiguous(), s.contiguous()


def _quantize(x, layout):
    if layout == "rows":
        return _q_vec(x)
    if layout == "cols":
        return _q_vec(x.transpose(-1, -2))
    return _q_blk(x if layout == "blocks" else x.transpose(-1, -2))


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _heavy(g, R, C, dtype=torch.float32):
    """Activations: normal, with a size of its own for every row and a few large columns."""
    x = torch.randn(R, C, generator=g, device="cuda")
    x *= torch.exp(torch.randn(R, 1, generator=g, device="cuda"))
    x *= 1 + 10 * (torch.rand(1, C, generator=g, device="cuda") < 0.01)
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    op = case["op"]
    if op == "quantize":
        dt = DT[case["dtype"]]
        shape = (case["G"], case["R"], case["C"]) if case["G"] > 1 else (case["R"], case["C"])
        x = _heavy(g, math.prod(shape[:-1]), shape[-1], dt).view(shape)
        return dict(case=case, x=x)
    if op == "gemm":
        rows = _counts(case)
        off = _regions(rows)
        M = case["rows"] if case["n"] == 1 else off[-1] + case["slack"]
        x = torch.zeros(M, case["K"], device="cuda")
        for r0, r in zip(off, rows):
            x[r0:r0 + r] = _heavy(g, r, case["K"])
        A, sa = _q_vec(x)
        W, sw = _q_blk(_normal(g, case["n"], case["N"], case["K"], std=case["K"] ** -0.5))
        st = dict(case=case, A=A, sa=sa, W=W, sw=sw, off=off,
                  offsets=torch.tensor(off, dtype=torch.int32, device="cuda") if case["n"] > 1 else None,
                  C=torch.zeros(M, case["N"], dtype=DT[case["out"]], device="cuda"))
        if own:
            import paper_2503_02495_b200 as uoe
            st["prob"] = uoe.Fp8Problem(n=case["n"], M=M, N=case["N"], K=case["K"], dtype=case["out"])
            st["ws"] = uoe.alloc_fp8_workspace(st["prob"])
        return st
    if op == "wgrad":
        rows = _counts(case)
        off = _regions(rows)
        K = max(off[-1], BLOCK)
        x, dy = torch.zeros(K, case["M"], device="cuda"), torch.zeros(K, case["N"], device="cuda")
        for r0, r in zip(off, rows):
            x[r0:r0 + r] = _heavy(g, r, case["M"])
            dy[r0:r0 + r] = _normal(g, r, case["N"], std=0.01)
        A, sa = _quantize(x, "cols")
        Bq, sb = _quantize(dy, "cols")
        st = dict(case=case, A=A, sa=sa, Bq=Bq, sb=sb, off=off, offsets=torch.tensor(off, dtype=torch.int32, device="cuda"),
                  dW=torch.empty(case["n"], case["M"], case["N"], device="cuda"))
        if own:
            import paper_2503_02495_b200 as uoe
            st["prob"] = uoe.Fp8Problem(n=case["n"], M=case["M"], N=case["N"], K=K, dtype="f32")
            st["ws"] = uoe.alloc_fp8_workspace(st["prob"])
        return st
    # the two layers
    n, d, d_e, k = case["n"], case["d"], case["d_e"], case["k"]
    wt = case.get("weights", "fp8")
    dt = torch.float32 if wt == "f32" else torch.bfloat16
    st = dict(case=case, Wr=_normal(g, d, n, std=4.0 * d ** -0.5, dtype=dt))
    W1, W2 = _normal(g, n, d, d_e, std=d ** -0.5, dtype=dt), _normal(g, n, d_e, d, std=d_e ** -0.5, dtype=dt)
    if wt == "fp8":
        (st["W1"], st["s1"]), (st["W2"], st["s2"]) = _quantize(W1, "blocks_t"), _quantize(W2, "blocks_t")
    else:
        st.update(W1=W1, W2=W2, s1=None, s2=None)
    st["b1"] = _normal(g, n, d_e, std=0.1, dtype=dt) if case["bias"] else None
    st["b2"] = _normal(g, n, d, std=0.1, dtype=dt) if case["bias"] else None
    if op == "tokens":
        st["x"] = _heavy(g, case["T"], d, dt)
        st["x"] = (st["x"].float() * torch.rsqrt((st["x"].float() ** 2).mean(-1, keepdim=True) + 1e-6)).to(dt)
        if own:
            import paper_2503_02495_b200 as uoe
            p = uoe.Problem(B=case["T"], L=1, L_valid=1, d=d, n=n, k=k, m=1, c=1, d_e=d_e, dtype="f32" if wt == "f32" else "bf16",
                            act=case["act"], gate=case["gate"])
            st.update(prob=p, r=uoe.alloc_routing(p), ws=uoe.alloc_workspace(p, uoe.UOE_OP_MLP_TOKENS), y=torch.empty_like(st["x"]))
        return st
    B, m, c, l_p = case["B"], case["m"], case["c"], case["l_p"]
    L, Lv = m * l_p, case["L_valid"]
    x = _normal(g, B, L, d)
    x[:, Lv:] = 0
    st["x"] = x.to(dt)
    real = _ceil(Lv, l_p)
    # a routing: experts drawn with Zipf weights, patches at random, both ascending; unused slots -1
    lean = -torch.log(torch.arange(1, n + 1, device="cuda").float())
    noise = -torch.log(-torch.log(torch.rand(B, n, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    e = (lean + noise).topk(k, 1).indices.sort(1).values
    cc = min(c, real)
    p = torch.rand(B, k, real, generator=g, device="cuda").topk(cc, 2).indices.sort(2).values
    patch = torch.full((B, k, c), -1, dtype=torch.int64, device="cuda")
    patch[..., :cc] = p
    gate = torch.rand(B, k, c, generator=g, device="cuda") * (patch >= 0)
    cnt = [int(v) for v in torch.bincount(e.flatten(), minlength=n).tolist()]
    off = _regions([q * c * l_p for q in cnt])
    st.update(expert_idx=e.int(), patch_idx=patch.int().contiguous(), gate=gate if case["gate"] else torch.ones_like(gate) * (patch >= 0),
              off=off, offsets=torch.tensor(off, dtype=torch.int32, device="cuda"))
    # the rows of every expert, for the plain form: (sample, position) of its tokens
    st["tok"], st["w"] = [], []
    for i in range(n):
        b, s = (e == i).nonzero(as_tuple=True)
        pj = patch[b, s]                                                   # [pairs, c]
        t = (pj * l_p).unsqueeze(-1) + torch.arange(l_p, device="cuda")
        ok = (pj >= 0).unsqueeze(-1) & (t < Lv)
        st["tok"].append((b.view(-1, 1, 1) * L + t)[ok])
        st["w"].append(st["gate"][b, s].unsqueeze(-1).expand_as(t)[ok])
    if own:
        import paper_2503_02495_b200 as uoe
        pr = uoe.Problem(B=B, L=L, L_valid=Lv, d=d, n=n, k=k, m=m, c=c, d_e=d_e, act=case["act"], gate=case["gate"])
        st.update(prob=pr, ws=uoe.alloc_workspace(pr, uoe.UOE_OP_MLP_FWD_FP8), y=torch.empty_like(st["x"]),
                  r=uoe.Routing(st["expert_idx"], st["patch_idx"], st["gate"], None, None, st["offsets"]))
    return st


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------

def _expand_vec(q, s):
    """Values of an operand with a scale per row and 128 columns: q [R, Cp], s [Cb, R]."""
    return (q.float().unflatten(-1, (-1, BLOCK)) * s.t().unsqueeze(-1)).flatten(-2)


def _expand_blk(q, s):
    """Values of an operand with a scale per 128 x 128 block: q [R, Cp], s [Rb, Cb]."""
    rows = s.repeat_interleave(BLOCK, 0)[:q.shape[0]]
    return (q.float().unflatten(-1, (-1, BLOCK)) * rows.unsqueeze(-1)).flatten(-2)


def _phi(h, act):
    if act == "silu":
        return h / (1 + torch.exp(-h))
    if act == "gelu_erf":
        return 0.5 * h * (1 + torch.erf(h * 2 ** -0.5))
    return 0.5 * h * (1 + torch.tanh((2 / math.pi) ** 0.5 * (h + 0.044715 * h ** 3)))


def _weight(st, name, i, K):
    """Values of expert i's weights as [out, K]."""
    if st["s" + name] is None:
        return st["W" + name][i].float().t()
    return _expand_blk(st["W" + name][i], st["s" + name][i])[:, :K]


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        import paper_2503_02495_b200 as uoe
        if op == "quantize":
            return uoe.uoe_fp8_quantize(st["x"], case["layout"])
        if op == "gemm":
            return uoe.uoe_fp8_gemm(st["prob"], st["A"], st["sa"], st["W"], st["sw"], st["offsets"], C=st["C"], ws=st["ws"], check=False)
        if op == "wgrad":
            return uoe.uoe_fp8_wgrad(st["prob"], st["A"], st["sa"], st["Bq"], st["sb"], st["offsets"], dW=st["dW"], ws=st["ws"], check=False)
        if op == "mlp":
            return uoe.uoe_mlp_forward_fp8(st["prob"], st["x"], st["W1"], st["s1"], st["W2"], st["s2"], st["r"], b1=st["b1"], b2=st["b2"],
                                           y=st["y"], ws=st["ws"], check=False)
        y = uoe.uoe_mlp_tokens(st["prob"], st["x"], st["Wr"], st["W1"], st["W2"], s1=st["s1"], s2=st["s2"], b1=st["b1"], b2=st["b2"],
                               r=st["r"], y=st["y"], ws=st["ws"], check=False)
        return y, st["r"].expert_idx
    if op == "quantize":
        return _quantize(st["x"], case["layout"])
    if op == "gemm":
        A = _expand_vec(st["A"], st["sa"])
        off = st["off"] if case["n"] > 1 else [0, A.shape[0]]
        for i in range(case["n"]):
            if off[i + 1] > off[i]:
                st["C"][off[i]:off[i + 1]] = A[off[i]:off[i + 1]] @ _expand_blk(st["W"][i], st["sw"][i]).t()
        return st["C"]
    if op == "wgrad":
        A, Bv = _expand_vec(st["A"], st["sa"]), _expand_vec(st["Bq"], st["sb"])
        for i in range(case["n"]):
            lo, hi = st["off"][i], st["off"][i + 1]
            st["dW"][i] = A[:, lo:hi] @ Bv[:, lo:hi].t()
        return st["dW"]
    n, d, d_e, k = case["n"], case["d"], case["d_e"], case["k"]
    if op == "mlp":
        x = st["x"].float().reshape(-1, d)
        y = x.clone()
        for i in range(n):
            if st["tok"][i].numel() == 0:
                continue
            h = _expand_vec(*_q_vec(x[st["tok"][i]]))[:, :d] @ _weight(st, "1", i, d).t()
            if st["b1"] is not None:
                h = h + st["b1"][i].float()
            z = _expand_vec(*_q_vec(_phi(h, case["act"])))[:, :d_e] @ _weight(st, "2", i, d_e).t()
            if st["b2"] is not None:
                z = z + st["b2"][i].float()
            y.index_add_(0, st["tok"][i], st["w"][i].unsqueeze(1) * z)
        return y.view(st["x"].shape).to(st["x"].dtype)
    x = st["x"].float()
    p = torch.softmax(st["x"].double() @ st["Wr"].double(), 1)
    e = p.sort(dim=1, descending=True, stable=True).indices[:, :k].sort(1).values
    y = x.clone()
    for i in range(n):
        t = (e == i).any(1).nonzero().flatten()
        if t.numel() == 0:
            continue
        h = x[t] @ _weight(st, "1", i, d).t()
        if st["b1"] is not None:
            h = h + st["b1"][i].float()
        z = _phi(h, case["act"]) @ _weight(st, "2", i, d_e).t()
        if st["b2"] is not None:
            z = z + st["b2"][i].float()
        w = p[t, i].float() ** 2 if case["gate"] else torch.ones(t.numel(), device=x.device)
        y.index_add_(0, t, w.unsqueeze(1) * z)
    return y.to(st["x"].dtype), e.int()


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "quantize":
        el = case["G"] * case["R"] * case["C"]
        per = BLOCK if case["layout"] in ("rows", "cols") else BLOCK * BLOCK
        return {"bytes": el * ((2 if case["dtype"] == "bf16" else 4) + 1) + 4 * el // per, "flops": 3 * el}
    if op in ("gemm", "wgrad"):
        R = case["rows"]
        if op == "gemm":
            N, K = case["N"], case["K"]
            used = sum(1 for r in _counts(case) if r)
            return {"bytes": R * K * (1 + 4 / BLOCK) + used * N * K + R * N * (2 if case["out"] == "bf16" else 4), "flops": 2 * R * N * K}
        M, N = case["M"], case["N"]
        return {"bytes": R * (M + N) * (1 + 4 / BLOCK) + case["n"] * M * N * 4, "flops": 2 * R * M * N}
    n, d, d_e, k = case["n"], case["d"], case["d_e"], case["k"]
    if op == "mlp":
        real = _ceil(case["L_valid"], case["l_p"])
        R = case["B"] * k * min(case["c"], real) * case["l_p"]
        return {"bytes": 2 * case["B"] * case["m"] * case["l_p"] * d * 2 + 2 * n * d * d_e, "flops": 4 * R * d * d_e}
    T = case["T"]
    used = n * (1 - (1 - k / n) ** T)                       # experts that T tokens choose, on average
    s = {"fp8": 1, "bf16": 2, "f32": 4}[case["weights"]]
    s_x = 4 if case["weights"] == "f32" else 2
    return {"bytes": used * 2 * d * d_e * s + (2 * T * d + d * n) * s_x, "flops": T * k * 4 * d * d_e + 2 * T * d * n}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------

def _e4m3(v):
    """The e4m3 value nearest to v (ties to even), |v| <= 448: steps of 2^(exponent - 3), the exponent at least -6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    step = torch.where(v.abs() >= step * 16, step * 2, step)
    step = torch.where((v.abs() < step * 8) & (step > 2.0 ** -9), step / 2, step)
    return torch.round(v / step) * step


def _quantize64(x, rows_per, cols_per):
    """(values in e4m3 [R, Cp], scale [R / rows_per, Cp / cols_per]) of x [R, C] in 64 bits."""
    R, C = x.shape
    p = torch.zeros(_ceil(R, rows_per) * rows_per, _ceil(C, cols_per) * cols_per, dtype=torch.float64, device=x.device)
    p[:R, :C] = x
    t = p.view(p.shape[0] // rows_per, rows_per, p.shape[1] // cols_per, cols_per)
    top = torch.clamp(t.abs().amax(dim=(1, 3)), min=2.0 ** -100)
    s = torch.exp2(torch.round(torch.log2(top / 448)) - 1)          # at most the power sought: raised until amax <= 448 s
    for _ in range(2):
        s = torch.where(top > 448 * s, 2 * s, s)
    return _e4m3(t / s[:, None, :, None]).reshape(p.shape)[:R], s


def _act64(h, act):
    if act == "silu":
        return h * torch.sigmoid(h)
    return torch.nn.functional.gelu(h, approximate="none" if act == "gelu_erf" else "tanh")


def _blocks64(q, s):
    out = q.double().clone()
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            out[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK] *= s[i, j].double()
    return out


def exact(case, seed):
    op = case["op"]
    st = prepare(case, seed)
    if op == "quantize":
        x = st["x"].double()
        x = x.unsqueeze(0) if x.dim() == 2 else x
        qs, ss = [], []
        for m in x:
            m = m.t() if case["layout"] in ("cols", "blocks_t") else m
            q, s = _quantize64(m, 1 if case["layout"] in ("rows", "cols") else BLOCK, BLOCK)
            qs.append(q)
            ss.append(s.t() if case["layout"] in ("rows", "cols") else s)
        q, s = torch.stack(qs), torch.stack(ss)
        return (q, s) if case["G"] > 1 else (q[0], s[0])
    if op == "gemm":
        out = torch.zeros(st["C"].shape, dtype=torch.float64, device="cuda")
        bounds = st["off"] if case["n"] > 1 else [0, case["rows"]]
        scale = st["sa"].double().t().repeat_interleave(BLOCK, 1)
        for i in range(case["n"]):
            lo, hi = bounds[i], bounds[i + 1]
            out[lo:hi] = torch.einsum("rk,jk->rj", st["A"][lo:hi].double() * scale[lo:hi], _blocks64(st["W"][i], st["sw"][i]))
        return out
    if op == "wgrad":
        out = torch.zeros(case["n"], case["M"], case["N"], dtype=torch.float64, device="cuda")
        for i in range(case["n"]):
            cols = slice(st["off"][i], st["off"][i + 1])
            blk = slice(st["off"][i] // BLOCK, st["off"][i + 1] // BLOCK)
            a = st["A"][:, cols].double() * st["sa"][blk].double().t().repeat_interleave(BLOCK, 1)
            b = st["Bq"][:, cols].double() * st["sb"][blk].double().t().repeat_interleave(BLOCK, 1)
            out[i] = torch.einsum("ir,jr->ij", a, b)
        return out
    x = st["x"].double()
    x = x.reshape(-1, x.shape[-1])
    mats = []
    for name in ("1", "2"):
        w, s = st["W" + name], st["s" + name]
        mats.append([w[i].double() if s is None else _blocks64(w[i], s[i]).t() for i in range(case["n"])])
    W1 = [w[:case["d"]] for w in mats[0]]
    W2 = [w[:case["d_e"]] for w in mats[1]]
    b1, b2 = st["b1"], st["b2"]
    y = x.clone()
    if op == "tokens":
        score = x @ st["Wr"].double()
        prob = torch.exp(score - score.amax(1, keepdim=True))
        prob /= prob.sum(1, keepdim=True)
    for i in range(case["n"]):
        if op == "tokens":
            # expert i is chosen where fewer than k experts come before it (larger, or equal with a lower index)
            before = (prob > prob[:, i:i + 1]).sum(1) + (prob[:, :i] == prob[:, i:i + 1]).sum(1)
            rows = (before < case["k"]).nonzero().flatten()
            weight = prob[rows, i] ** 2 if case["gate"] else torch.ones(len(rows), dtype=torch.float64, device="cuda")
            v = x[rows]
        else:
            rows, weight = st["tok"][i], st["w"][i].double()
            if len(rows) == 0:
                continue
            q, s = _quantize64(x[rows], 1, BLOCK)
            v = (q * s.repeat_interleave(BLOCK, 1))[:, :case["d"]]
        h = v @ W1[i] + (0 if b1 is None else b1[i].double())
        a = _act64(h, case["act"])
        if op == "mlp":
            q, s = _quantize64(a, 1, BLOCK)
            a = (q * s.repeat_interleave(BLOCK, 1))[:, :case["d_e"]]
        z = a @ W2[i] + (0 if b2 is None else b2[i].double())
        y.index_add_(0, rows, weight[:, None] * z)
    if op == "tokens":
        return y, None
    return y.view(st["x"].shape)
