"""GPU parity: uoe_fp8_quantize, uoe_fp8_gemm and uoe_fp8_wgrad against plain implementations in float64.

Quantisation is exact up to its one rounding, which both sides do on the same exact quotient: values and scales must be equal.
Products: the operands are exact on both sides (e4m3 values times float32 scales, formed in float64 by the reference), so the kernel's
error is its float32 arithmetic and the rounding of the result.  Per element of the sum: one product of two e4m3 values (exact in float32:
2 x 4 bits), at most 128 additions in the tensor core and Kb additions outside it, two roundings of the scales' product.  (With scales
that are powers of two the tensor core adds all of K, 32 products a step.)  With gamma = (128 + 4 Kb + 4) 2^-23 (a tensor-core addition counted
as truncating: one step of float32) the error is at most
gamma * sum |a| |b|; bfloat16 results add half a step, 2^-8 of the result.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BLOCK = 128


def _blk(v):
    return -(-v // BLOCK)


def _rand(seed, *shape, dtype=torch.float32, wide=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g, dtype=torch.float64)
    if wide:      # rows and columns of very different sizes
        x = x * torch.exp2(torch.randint(-12, 12, (*shape[:-1], 1), generator=g).double())
        x[..., ::37] *= 300
    return x.to(dtype)


def _e4m3_nearest(v):
    """Nearest e4m3 value, ties to even, from the list of all of them (float64, |v| <= 448)."""
    codes = torch.arange(127, dtype=torch.int64)
    e, m = codes >> 3, (codes & 7).double()
    vals = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2((e - 7).double()))
    a = v.abs().contiguous()
    hi = torch.searchsorted(vals, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - vals[lo], vals[hi] - a
    take_hi = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return torch.where(take_hi, vals[hi], vals[lo]) * torch.sign(v)


def _quantize_ref(x, rows_per):
    """x [R, C] float64 -> values [R, Cp], scale [R / rows_per, Cb]."""
    R, C = x.shape
    Rb, Cb = -(-R // rows_per), _blk(C)
    p = torch.zeros(Rb * rows_per, Cb * BLOCK, dtype=torch.float64)
    p[:R, :C] = x
    t = p.view(Rb, rows_per, Cb, BLOCK)
    top = t.abs().amax((1, 3)).clamp(min=2.0 ** -100)
    s = torch.exp2(torch.ceil(torch.log2(top / 448)))
    s = torch.where(top > 448 * s, s * 2, s)
    s = torch.where(top <= 448 * (s / 2), s / 2, s)
    return _e4m3_nearest(t / s[:, None, :, None]).reshape(Rb * rows_per, -1)[:R], s


def _layout_ref(x, layout):
    x = x.double()
    m = x.t() if layout in ("cols", "blocks_t") else x
    q, s = _quantize_ref(m.contiguous(), 1 if layout in ("rows", "cols") else BLOCK)
    return q, s.t() if layout in ("rows", "cols") else s


SIZES = [(1, 1), (3, 7), (128, 128), (129, 257), (200, 1000), (1, 4096), (777, 8), (64, 130), (300, 516)]


@pytest.mark.parametrize("layout", ["rows", "cols", "blocks", "blocks_t"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", SIZES)
def test_quantize(layout, dtype, size):
    import paper_2503_02495_b200 as uoe
    x = _rand(3, *size, dtype=dtype, wide=True)
    q, s = uoe.uoe_fp8_quantize(x.cuda(), layout)
    qr, sr = _layout_ref(x, layout)
    assert torch.equal(s.double().cpu(), sr)
    assert torch.equal(q.float().double().cpu(), qr)


@pytest.mark.parametrize("layout", ["rows", "cols", "blocks", "blocks_t"])
def test_quantize_several_matrices_and_special_values(layout):
    import paper_2503_02495_b200 as uoe
    x = _rand(5, 3, 150, 270)
    x[0, :130] = 0                                  # blocks of zeros
    x[1] *= 1e-38                                   # below the smallest scale: everything rounds to zero
    x[2, 3, 5] = 3e38
    x[2, 140, 200] = 448.0                          # the largest value itself keeps its scale
    q, s = uoe.uoe_fp8_quantize(x.cuda(), layout)
    for i in range(3):
        qr, sr = _layout_ref(x[i], layout)
        assert torch.equal(s[i].double().cpu(), sr) and torch.equal(q[i].float().double().cpu(), qr)


@pytest.mark.parametrize("layout", ["rows", "cols", "blocks", "blocks_t"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_quantize_a_block_without_a_finite_maximum(layout, bad):
    """Its scale is NaN and its values zeros; every other block is what it is without it."""
    import paper_2503_02495_b200 as uoe
    x = _rand(6, 200, 300)
    ref_q, ref_s = uoe.uoe_fp8_quantize(x.cuda(), layout)
    x[130, 140] = bad
    q, s = uoe.uoe_fp8_quantize(x.cuda(), layout)
    r, c = (130, 140) if layout in ("rows", "blocks") else (140, 130)
    at = (c // BLOCK, r) if layout in ("rows", "cols") else (r // BLOCK, c // BLOCK)
    rows = slice(r, r + 1) if layout in ("rows", "cols") else slice(r // BLOCK * BLOCK, (r // BLOCK + 1) * BLOCK)
    cols = slice(c // BLOCK * BLOCK, (c // BLOCK + 1) * BLOCK)
    assert torch.isnan(s[at])
    assert (q.float()[rows, cols] == 0).all()
    s[at] = ref_s[at]
    qf, rf = q.float(), ref_q.float()
    qf[rows, cols] = rf[rows, cols]
    assert torch.equal(qf, rf) and torch.equal(s, ref_s)


def test_quantize_into_given_tensors_keeps_what_lies_behind():
    import paper_2503_02495_b200 as uoe
    x = _rand(8, 130, 200)
    buf = torch.full((130 * 256 + 512,), 7, dtype=torch.uint8, device="cuda")
    q = buf[:130 * 256].view(torch.float8_e4m3fn).view(130, 256)
    uoe.uoe_fp8_quantize(x.cuda(), "rows", q=q)
    assert (buf[130 * 256:] == 7).all()
    assert (q.float()[:, 200:] == 0).all()


# ------------------------------------------------------------------------------------------------------------------
# products
# ------------------------------------------------------------------------------------------------------------------

def _vec_values(q, s):
    return q.float().double() * s.double().t().repeat_interleave(BLOCK, 1)


def _blk_values(q, s):
    return q.float().double() * s.double().repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)


def _gamma(Kb):
    return (128 + 4 * Kb + 4) * 2.0 ** -23


def _regions(counts):
    off = [0]
    for c in counts:
        off.append(off[-1] + _blk(c) * BLOCK)
    return off


def _close(got, ref, bound, dtype):
    tol = bound + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 2.0 ** -24 * ref.abs()) + 1e-37
    bad = ~((got.double().cpu() - ref).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((got.double().cpu() - ref).abs() / tol).max()))


GEMMS = {
    "one": dict(counts=[1], N=1, K=1),
    "one_token": dict(counts=[1], N=512, K=512),
    "one_token_odd": dict(counts=[1], N=333, K=700),
    "four_tokens": dict(counts=[4], N=300, K=1000),
    "seventeen_tokens": dict(counts=[17], N=136, K=300),
    "sixty_five": dict(counts=[65], N=264, K=140),
    "tile": dict(counts=[128], N=128, K=128),
    "odd": dict(counts=[333], N=77, K=129),
    "wide": dict(counts=[1000], N=1000, K=384),
    "long": dict(counts=[130], N=130, K=5000),
    "split": dict(counts=[250], N=300, K=9000),
    "split_experts": dict(counts=[200, 0, 70], slack=40, N=140, K=3300),
    "experts": dict(counts=[100, 0, 300, 1], slack=130, N=200, K=260),
    "pairs": dict(counts=[5000, 128, 4100, 0, 3000, 129], slack=300, N=1030, K=640),
    "experts_wide_tiles": dict(counts=[2000, 3500, 129, 0, 4000], slack=1, N=1030, K=512),
    "all_empty": dict(counts=[0, 0, 0], slack=200, N=64, K=64),
    "thirty_two": dict(counts=[5] * 32, N=40, K=48),
}


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(GEMMS))
def test_gemm(name, out, any_scale):
    import paper_2503_02495_b200 as uoe
    c = GEMMS[name]
    n, N, K = len(c["counts"]), c["N"], c["K"]
    off = _regions(c["counts"])
    M = c["counts"][0] if n == 1 else off[-1] + c.get("slack", 0)
    x = torch.zeros(M, K)
    for o, cnt in zip(off, c["counts"]):
        x[o:o + cnt] = _rand(o + 1, cnt, K, wide=True)
    W = _rand(2, n, N, K)
    A, sa = uoe.uoe_fp8_quantize(x.cuda(), "rows")
    Wq, sw = uoe.uoe_fp8_quantize(W.cuda(), "blocks")
    g = torch.Generator().manual_seed(9)
    if any_scale:                                                   # scales that are no powers of two
        sa *= (0.5 + torch.rand(sa.shape, generator=g)).cuda()
        sw *= (0.5 + torch.rand(sw.shape, generator=g)).cuda()
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    C = torch.full((M, N), -3.0, dtype=dt, device="cuda")
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda") if n > 1 else None
    prob = uoe.Fp8Problem(n=n, M=M, N=N, K=K, dtype=out, any_scale=any_scale)
    got = uoe.uoe_fp8_gemm(prob, A, sa, Wq, sw, offsets, C=C)
    a = _vec_values(A.cpu(), sa.cpu())
    bounds = off if n > 1 else [0, M]
    for e in range(n):
        w = _blk_values(Wq[e].cpu(), sw[e].cpu())
        lo, hi = bounds[e], bounds[e + 1]
        _close(got[lo:hi], a[lo:hi] @ w.t(), _gamma(_blk(K)) * (a[lo:hi].abs() @ w.abs().t()), out)
    assert (got[bounds[n]:] == -3).all()
    assert torch.equal(got, uoe.uoe_fp8_gemm(prob, A, sa, Wq, sw, offsets, C=torch.full_like(C, -3)))      # the same bits each time


WGRADS = {
    "one": dict(counts=[1], M=8, N=8),
    "odd": dict(counts=[130, 0, 400, 1], M=77, N=333),
    "wide": dict(counts=[3000, 1000, 2500], M=1100, N=600),
    "pairs": dict(counts=[300, 0, 128, 500, 1000, 129, 1, 700], M=1300, N=1000),
    "many_tiles": dict(counts=[300, 0, 128, 500], M=1024, N=2304),
    "split": dict(counts=[6500, 1], M=130, N=77),
    "empty": dict(counts=[0, 0], M=40, N=24),
}


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("name", list(WGRADS))
def test_wgrad(name, any_scale):
    import paper_2503_02495_b200 as uoe
    c = WGRADS[name]
    n, M, N = len(c["counts"]), c["M"], c["N"]
    off = _regions(c["counts"])
    K = max(off[-1], 128)
    x, dy = torch.zeros(K, M), torch.zeros(K, N)
    for o, cnt in zip(off, c["counts"]):
        x[o:o + cnt], dy[o:o + cnt] = _rand(o + 1, cnt, M, wide=True), _rand(o + 2, cnt, N)
    A, sa = uoe.uoe_fp8_quantize(x.cuda(), "cols")
    B, sb = uoe.uoe_fp8_quantize(dy.cuda(), "cols")
    g = torch.Generator().manual_seed(9)
    if any_scale:
        sa *= (0.5 + torch.rand(sa.shape, generator=g)).cuda()
        sb *= (0.5 + torch.rand(sb.shape, generator=g)).cuda()
    prob = uoe.Fp8Problem(n=n, M=M, N=N, K=K, dtype="f32", any_scale=any_scale)
    dW = torch.full((n, M, N), -3.0, device="cuda")
    got = uoe.uoe_fp8_wgrad(prob, A, sa, B, sb, torch.tensor(off, dtype=torch.int32, device="cuda"), dW=dW)
    a, b = _vec_values(A.cpu(), sa.cpu()), _vec_values(B.cpu(), sb.cpu())
    for e in range(n):
        ae, be = a[:, off[e]:off[e + 1]], b[:, off[e]:off[e + 1]]
        _close(got[e], ae @ be.t(), _gamma(_blk(c["counts"][e])) * (ae.abs() @ be.abs().t()), "f32")


def test_offsets_of_another_form_are_reported():
    import paper_2503_02495_b200 as uoe
    x, W = _rand(1, 512, 64).cuda(), _rand(2, 2, 64, 64).cuda()
    A, sa = uoe.uoe_fp8_quantize(x, "rows")
    Wq, sw = uoe.uoe_fp8_quantize(W, "blocks")
    prob = uoe.Fp8Problem(n=2, M=512, N=64, K=64)
    for off in ([0, 100, 256], [0, 256, 128], [0, 256, 640], [-128, 0, 256]):
        C = torch.full((512, 64), -3.0, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(uoe.UoeError) as ei:
            uoe.uoe_fp8_gemm(prob, A, sa, Wq, sw, torch.tensor(off, dtype=torch.int32, device="cuda"), C=C)
        assert ei.value.status == 6
        assert (C == -3).all()


def test_a_row_with_a_nan_spoils_only_itself():
    import paper_2503_02495_b200 as uoe
    x, W = _rand(1, 256, 300), _rand(2, 1, 64, 300)
    ref = None
    for bad in (False, True):
        if bad:
            x[70, 299] = float("nan")
        A, sa = uoe.uoe_fp8_quantize(x.cuda(), "rows")
        Wq, sw = uoe.uoe_fp8_quantize(W.cuda(), "blocks")
        got = uoe.uoe_fp8_gemm(uoe.Fp8Problem(n=1, M=256, N=64, K=300), A, sa, Wq, sw)
        if bad:
            assert torch.isnan(got[70]).all()
            got[70] = ref[70]
            assert torch.equal(got, ref)
        ref = got


def test_a_scale_that_is_no_power_of_two_is_reported():
    import paper_2503_02495_b200 as uoe
    A, sa = uoe.uoe_fp8_quantize(_rand(1, 200, 300).cuda(), "rows")
    W, sw = uoe.uoe_fp8_quantize(_rand(2, 1, 64, 300).cuda(), "blocks")
    prob = uoe.Fp8Problem(n=1, M=200, N=64, K=300)
    ref = uoe.uoe_fp8_gemm(prob, A, sa, W, sw)
    for bad in (0.75, 0.0, -1.0, 2.0 ** -130):
        s2 = sa.clone()
        s2[1, 150] = bad
        C, ws = torch.empty_like(ref), uoe.alloc_fp8_workspace(prob)
        uoe.uoe_fp8_gemm(prob, A, s2, W, sw, C=C, ws=ws, check=False)
        assert uoe.uoe_read_device_status(ws) == 8 and "power of two" in uoe.status_string(8)
        assert torch.isnan(C[150]).all()
        C[150] = ref[150]
        assert torch.equal(C, ref)


@pytest.mark.parametrize("counts, N, K, any_scale", [([3], 300, 1000, False), ([250], 300, 9000, False), ([300, 0, 500], 200, 260, True),
                                                     ([5000, 128, 4100], 1030, 640, False)])
def test_captured_and_on_two_streams(counts, N, K, any_scale):
    """Quantisation, product and weight gradient in one graph: replays follow what is in x; two streams with a workspace each do not meet."""
    import paper_2503_02495_b200 as uoe
    n, off = len(counts), _regions(counts)
    M = counts[0] if n == 1 else off[-1]
    live = torch.zeros(M, 1)
    for o, cnt in zip(off, counts):
        live[o:o + cnt] = 1
    xs = [(_rand(3 + i, M, K) * live).cuda() for i in range(2)]
    dy = (_rand(7, M, N) * live).cuda()
    W, sw = uoe.uoe_fp8_quantize(_rand(2, n, N, K).cuda(), "blocks")
    o = torch.tensor(off, dtype=torch.int32, device="cuda") if n > 1 else None
    prob = uoe.Fp8Problem(n=n, M=M, N=N, K=K, any_scale=any_scale)
    wprob = uoe.Fp8Problem(n=n, M=K, N=N, K=M, dtype="f32", any_scale=any_scale)

    def step(x, ws):
        A, sa = uoe.uoe_fp8_quantize(x, "rows")
        C = uoe.uoe_fp8_gemm(prob, A, sa, W, sw, o, ws=ws, check=False)
        return C[:off[-1]], uoe.uoe_fp8_wgrad(wprob, *uoe.uoe_fp8_quantize(x, "cols"), *uoe.uoe_fp8_quantize(dy, "cols"), o, ws=ws, check=False)

    wss = [uoe.alloc_fp8_workspace(prob) for _ in range(2)]
    want = [[t.clone() for t in step(x, wss[0])] for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [None, None]
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = step(xs[i], wss[i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    held = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(held, wss[0])
    for i in (0, 1, 0):
        held.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))


def test_offsets_that_pass_32_bits():
    """More than 2^32 bytes of input and 2^31 elements: the last rows are what they are alone."""
    import paper_2503_02495_b200 as uoe
    R, C = 2 ** 20 + 131, 2056
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    tail = _rand(4, 200, C, dtype=torch.bfloat16)
    x[-200:] = tail.cuda()
    for layout in ("rows", "cols"):
        q, s = uoe.uoe_fp8_quantize(x, layout)
        if layout == "rows":
            qr, sr = _layout_ref(tail, layout)
            assert torch.equal(q[-200:].float().double().cpu(), qr) and torch.equal(s[:, -200:].double().cpu(), sr)
        else:
            rest = R % BLOCK or BLOCK                                      # rows of the last block
            qr, sr = _layout_ref(tail[-rest:], layout)
            assert torch.equal(q[:, -BLOCK:][:, :rest].float().double().cpu(), qr[:, :rest]) and torch.equal(s[-1].double().cpu(), sr[0])
        del q, s
    del x
    A, sa = uoe.uoe_fp8_quantize(torch.cat([torch.zeros(R - 200, 24), tail[:, :24].float()]).cuda(), "rows")
    W, sw = uoe.uoe_fp8_quantize(_rand(5, 1, C, 24).cuda(), "blocks")
    got = uoe.uoe_fp8_gemm(uoe.Fp8Problem(n=1, M=R, N=C, K=24), A, sa, W, sw)[-200:]
    a, w = _vec_values(A[-200:].cpu(), sa[:, -200:].cpu()), _blk_values(W[0].cpu(), sw[0].cpu())
    _close(got, a @ w.t(), _gamma(1) * (a.abs() @ w.abs().t()), "bf16")
