"""GPU parity: operands of the 8-bit products as callers hold them.

A transposed operand holds the same values, so the product has the same bits; its values are moved, not computed, and are compared exactly.
"""
import pytest
import torch

from tests.test_gpu_fp8 import BLOCK, _blk_values, _close, _gamma, _rand, _regions, _vec_values

pytestmark = pytest.mark.gpu


def _turned(q):
    """The same values with the contraction not contiguous."""
    t = q.transpose(-1, -2).view(torch.uint8).contiguous().view(q.dtype).transpose(-1, -2)
    assert t.shape == q.shape and (1 in q.shape or not t.is_contiguous())
    return t


@pytest.mark.parametrize("G, R, C", [(1, 128, 1), (1, 128, 16), (1, 256, 77), (3, 384, 129), (2, 128, 1000), (1, 1280, 4096), (5, 256, 33)])
def test_transpose(G, R, C):
    import paper_2503_02495_b200 as uoe
    g = torch.Generator().manual_seed(R + C)
    x = torch.randint(0, 256, (G, R, C), generator=g, dtype=torch.uint8)
    buf = torch.full((G * R * C + 256,), 7, dtype=torch.uint8, device="cuda")
    q = buf[:G * R * C].view(G, C, R).view(torch.float8_e4m3fn)
    uoe.uoe_fp8_transpose(x.cuda().view(torch.float8_e4m3fn), q=q)
    assert torch.equal(q.view(torch.uint8).cpu(), x.transpose(1, 2)) and (buf[G * R * C:] == 7).all()


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("counts, M, N", [([1], 8, 8), ([130, 0, 400, 1], 77, 333), ([300, 0, 128, 500], 512, 256), ([3000, 1000], 1100, 600)])
def test_wgrad_of_operands_that_lie_the_other_way_round(counts, M, N, any_scale):
    """Operands quantised by columns and not turned, strides (1, M): against float64, and with the bits of the turned ones."""
    import paper_2503_02495_b200 as uoe
    off = _regions(counts)
    x, dy = torch.zeros(off[-1], M), torch.zeros(off[-1], N)
    for o, cnt in zip(off, counts):
        x[o:o + cnt], dy[o:o + cnt] = _rand(o + 1, cnt, M, wide=True), _rand(o + 2, cnt, N)
    A, sa = uoe.uoe_fp8_quantize(x.cuda(), "cols")
    B, sb = uoe.uoe_fp8_quantize(dy.cuda(), "cols")
    prob = uoe.Fp8Problem(n=len(counts), M=M, N=N, K=off[-1], dtype="f32", any_scale=any_scale)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    got = uoe.uoe_fp8_wgrad(prob, _turned(A), sa, _turned(B), sb, o)
    assert torch.equal(got, uoe.uoe_fp8_wgrad(prob, A, sa, B, sb, o))
    assert torch.equal(got, uoe.uoe_fp8_wgrad(prob, A, sa, _turned(B), sb, o))
    a, b = _vec_values(A.cpu(), sa.cpu()), _vec_values(B.cpu(), sb.cpu())
    for e, cnt in enumerate(counts):
        ae, be = a[:, off[e]:off[e + 1]], b[:, off[e]:off[e + 1]]
        _close(got[e], ae @ be.t(), _gamma(-(-cnt // BLOCK)) * (ae.abs() @ be.abs().t()), "f32")


@pytest.mark.parametrize("counts, N, K", [([3], 300, 1000), ([200, 0, 70], 140, 330)])
def test_gemm_of_operands_that_lie_the_other_way_round(counts, N, K):
    import paper_2503_02495_b200 as uoe
    n, off = len(counts), _regions(counts)
    M = counts[0] if n == 1 else off[-1]
    A, sa = uoe.uoe_fp8_quantize(_rand(1, M, K).cuda(), "rows")
    W, sw = uoe.uoe_fp8_quantize(_rand(2, n, N, K).cuda(), "blocks")
    o = torch.tensor(off, dtype=torch.int32, device="cuda") if n > 1 else None
    prob = uoe.Fp8Problem(n=n, M=M, N=N, K=K)
    got = uoe.uoe_fp8_gemm(prob, _turned(A), sa, _turned(W), sw, o)
    assert torch.equal(got, uoe.uoe_fp8_gemm(prob, A, sa, W, sw, o))
    a = _vec_values(A.cpu(), sa.cpu())
    for e in range(n):
        s = slice(off[e], off[e + 1] if n > 1 else M)
        w = _blk_values(W[e].cpu(), sw[e].cpu())
        _close(got[s], a[s] @ w.t(), _gamma(-(-K // BLOCK)) * (a[s].abs() @ w.abs().t()), "bf16")


def test_wgrad_of_turned_operands_captured():
    import paper_2503_02495_b200 as uoe
    q = [uoe.uoe_fp8_quantize(_rand(s, 256, c).cuda(), "cols") for s, c in ((1, 200), (2, 72))]
    (A, sa), (B, sb) = q
    At, Bt = _turned(A), _turned(B)
    prob = uoe.Fp8Problem(n=1, M=200, N=72, K=256, dtype="f32")
    ws = uoe.alloc_fp8_workspace(prob)
    want = uoe.uoe_fp8_wgrad(prob, A, sa, B, sb, ws=ws)
    dW = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uoe.uoe_fp8_wgrad(prob, At, sa, Bt, sb, dW=dW, ws=ws, check=False)
    for _ in range(2):
        dW.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dW, want)


@pytest.mark.parametrize("scale, status", [(float("inf"), 8), (-float("inf"), 8), (float("nan"), 0), (-float("nan"), 0)])
def test_a_scale_that_is_not_finite(scale, status):
    """NaN is what the quantisation writes for a block without a finite maximum, whatever its sign bit; an infinity is no power of two."""
    import math
    import paper_2503_02495_b200 as uoe
    A, sa = uoe.uoe_fp8_quantize(_rand(1, 200, 300).cuda(), "rows")
    W, sw = uoe.uoe_fp8_quantize(_rand(2, 1, 64, 300).cuda(), "blocks")
    prob = uoe.Fp8Problem(n=1, M=200, N=64, K=300)
    ref = uoe.uoe_fp8_gemm(prob, A, sa, W, sw)
    bits = {8: 0x7f800000, 0: 0x7fc00000}[status] | (0x80000000 if math.copysign(1, scale) < 0 else 0)
    sa.view(torch.int32)[1, 150] = bits - (1 << 32) if bits >> 31 else bits
    C, ws = torch.empty_like(ref), uoe.alloc_fp8_workspace(prob)
    uoe.uoe_fp8_gemm(prob, A, sa, W, sw, C=C, ws=ws, check=False)
    assert uoe.uoe_read_device_status(ws) == status
    assert torch.isnan(C[150]).all()
    C[150] = ref[150]
    assert torch.equal(C, ref)


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("rows, M", [(40, 40 + 88), (40, 300), (300, 600)])
def test_one_expert_with_offsets(rows, M, any_scale):
    """n = 1 with offsets: the region's rows and no others, whichever kernel would take all M of them."""
    import paper_2503_02495_b200 as uoe
    end = -(-rows // BLOCK) * BLOCK
    x = torch.zeros(M, 260)
    x[:rows] = _rand(1, rows, 260, wide=True)
    A, sa = uoe.uoe_fp8_quantize(x.cuda(), "rows")
    W, sw = uoe.uoe_fp8_quantize(_rand(2, 1, 140, 260).cuda(), "blocks")
    C = torch.full((M, 140), -3.0, device="cuda")
    prob = uoe.Fp8Problem(n=1, M=M, N=140, K=260, dtype="f32", any_scale=any_scale)
    uoe.uoe_fp8_gemm(prob, A, sa, W, sw, torch.tensor([0, end], dtype=torch.int32, device="cuda"), C=C)
    a, w = _vec_values(A.cpu(), sa.cpu())[:end], _blk_values(W[0].cpu(), sw[0].cpu())
    _close(C[:end], a @ w.t(), _gamma(3) * (a.abs() @ w.abs().t()), "f32")
    assert (C[end:] == -3).all()


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("counts, M, N", [([6500, 1], 130, 77), ([300, 0, 128, 500, 1000, 129, 1, 700], 1300, 1000), ([130, 0, 400, 1], 77, 333)])
def test_wgrad_has_the_same_bits_each_time(counts, M, N, any_scale):
    import paper_2503_02495_b200 as uoe
    off = _regions(counts)
    x, dy = torch.zeros(off[-1], M), torch.zeros(off[-1], N)
    for o, cnt in zip(off, counts):
        x[o:o + cnt], dy[o:o + cnt] = _rand(o + 1, cnt, M, wide=True), _rand(o + 2, cnt, N)
    q = [*uoe.uoe_fp8_quantize(x.cuda(), "cols"), *uoe.uoe_fp8_quantize(dy.cuda(), "cols")]
    prob = uoe.Fp8Problem(n=len(counts), M=M, N=N, K=off[-1], dtype="f32", any_scale=any_scale)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    ref = uoe.uoe_fp8_wgrad(prob, *q, o)
    for _ in range(5):
        assert torch.equal(ref, uoe.uoe_fp8_wgrad(prob, *q, o))
