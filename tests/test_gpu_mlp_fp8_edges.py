"""GPU parity: uoe_mlp_forward_fp8 where weights and values are no numbers, and gradients from the 8-bit products against differences."""
import pytest
import torch

from tests.helpers import to_dev
from tests.test_gpu_fp8 import BLOCK
from tests.test_gpu_mlp_fp8 import _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["by_patch", "several_tiles", "odd_widths"])
def test_padding_rows_keep_x_whatever_the_weights_of_their_patch(name, bad):
    """y = x on a sample's padding rows, also in a patch whose combine weight is no number."""
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, _), (W2, s2, _), b = _setup(name)
    last = w.m - 1
    hit = (r.patch_idx == last).nonzero()
    assert len(hit) and w.L_valid % w.l_p
    for q in hit.tolist():
        r.gate[tuple(q)] = bad
    xd = to_dev(x)
    got = uoe.uoe_mlp_forward_fp8(prob, xd, W1, s1, W2, s2, r)
    assert torch.equal(got[:, w.L_valid:], xd[:, w.L_valid:])
    rows = got[int(hit[0][0]), last * w.l_p:w.L_valid]
    assert not torch.isfinite(rows).any()


@pytest.mark.parametrize("name", ["by_patch", "several_tiles", "gathered_patches_of_8", "pairs_of_ctas", "any_scale", "odd_widths"])
def test_a_token_with_a_nan_spoils_only_itself(name):
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, _), (W2, s2, _), b = _setup(name)
    xd = to_dev(x)
    ref = uoe.uoe_mlp_forward_fp8(prob, xd, W1, s1, W2, s2, r)
    patch = int(r.patch_idx[1, 0, 0])
    t = patch * w.l_p + (w.l_p - 1) // 2                                   # a token that some expert takes
    assert t < w.L_valid
    xd[1, t, w.d // 2] = float("nan")
    got = uoe.uoe_mlp_forward_fp8(prob, xd, W1, s1, W2, s2, r)
    assert torch.isnan(got[1, t]).all()
    got[1, t] = ref[1, t]
    assert torch.equal(got, ref)


def test_gradients_against_differences():
    """<dy, C(x + t v) - C(x)> = t <dx, v> and <dy, C(W + t V) - C(W)> = t <dW, V>, the left sides in float64 on the dequantised operands (C is
    linear in each, so they are exact but for float64), the right sides from the library's dx and dW on the same operands.  dx is the product
    of dy and W, dW that of x and dy, each sum of K terms off by at most K 2^-23 sum |terms|; the sums over v and V are float64.  v and V go
    uphill (the gradient's signs, sizes of their own), so that nothing cancels: a gradient of zeros or of the other sign is far outside the bound."""
    import paper_2503_02495_b200 as uoe
    g = torch.Generator().manual_seed(6)
    n, K, N, off = 3, 200, 136, [0, 256, 256, 640]
    live = torch.zeros(640, 1)
    live[:200], live[256:600] = 1, 1
    x, dy = torch.randn(640, K, generator=g) * live, torch.randn(640, N, generator=g) * live
    W = torch.randn(n, K, N, generator=g) * K ** -0.5
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    q = lambda t, lay: uoe.uoe_fp8_quantize(t.cuda(), lay)
    rows = lambda qs, C: (qs[0].float().cpu().double() * qs[1].cpu().double().t().repeat_interleave(BLOCK, 1))[:, :C]
    Wb = q(W, "blocks")                                                    # [n, K, N], contracted over N: dx
    Wv = (Wb[0].float().cpu().double() * Wb[1].cpu().double().repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(BLOCK, 2))[..., :N]
    dr = q(dy, "rows")
    dx = uoe.uoe_fp8_gemm(uoe.Fp8Problem(n, 640, K, N, "f32"), *dr, *Wb, o).cpu().double()
    xc, dc = q(x, "cols"), q(dy, "cols")
    dW = uoe.uoe_fp8_wgrad(uoe.Fp8Problem(n, K, N, 640, "f32"), *xc, *dc, o).cpu().double()
    dyr = rows(dr, N)
    xv, dyc = (rows((qs[0], qs[1]), 640).t() for qs in (xc, dc))            # as dW's product holds them
    t = 0.5
    v, V = torch.rand(640, K, generator=g).double(), torch.rand(n, K, N, generator=g).double()
    for e in (0, 2):
        s = slice(off[e], off[e + 1])
        v[s] *= torch.sign(dyr[s] @ Wv[e].t())
        V[e] *= torch.sign(xv[s].t() @ dyc[s])
        left = (dyr[s] * ((xv[s] + t * v[s]) @ Wv[e] - xv[s] @ Wv[e])).sum()
        right = t * (dx[s] * v[s]).sum()
        room = t * N * 2.0 ** -23 * ((dyr[s].abs() @ Wv[e].abs().t()) * v[s].abs()).sum() + 1e-9
        assert (left - right).abs() <= room < 0.01 * left.abs()
        left = (dyc[s] * (xv[s] @ (Wv[e] + t * V[e]) - xv[s] @ Wv[e])).sum()
        right = t * (dW[e] * V[e]).sum()
        room = t * (off[e + 1] - off[e]) * 2.0 ** -23 * ((xv[s].abs().t() @ dyc[s].abs()) * V[e].abs()).sum() + 1e-9
        assert (left - right).abs() <= room < 0.01 * left.abs()
    assert (dW[1] == 0).all()
