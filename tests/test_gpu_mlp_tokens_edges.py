"""GPU parity: uoe_mlp_tokens where it can go wrong: hidden widths, values far out, infinities, what nobody chose, what a workspace held before.

References and bounds are those of test_gpu_mlp_tokens.py (float64, element by element) where nothing else is said.
"""
import pytest
import torch

from tests.test_gpu_mlp_tokens import _case, _check, make, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, d, d_e, bias", [(1, 64, 33, False), (1, 136, 1, True), (9, 72, 12, True), (20, 264, 130, False), (40, 128, 257, True), (64, 72, 7, False)])
def test_8_bit_weights_of_any_hidden_width(T, d, d_e, bias):
    """Rows of 8-bit weights are padded to 128, so no width is refused: what uoe_mlp_forward_fp8 takes for a prompt can be decoded."""
    import paper_2503_02495_b200 as uoe
    c = _case(T, d, d_e, 5, 2, "fp8", act="gelu_tanh", bias=bias)
    m = make(c)
    prob, call, v1, v2 = run(c, m)
    r = uoe.alloc_routing(prob)
    got = call(r=r)
    y, bound, e, _ = reference(c, m["x"], m["Wr"], v1, v2, m["b1"], m["b2"])
    assert torch.equal(r.expert_idx.cpu().long(), e)
    _check(got, y, bound)
    assert torch.equal(got, call())


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_float32_activation_keeps_its_bits(act):
    """phi alone (both layers the identity, no gate, no residual) over the whole range where it is not zero.

    SiLU h / (1 + e^-h): e^-h is off by 2 steps of float32 (2 x 2^-23 of it), the sum and the quotient by half a step each: 3 x 2^-23 of the
    result; from |h| = 88.7 on e^-h passes the largest float32, and the quotient, at most 89 / 3.4e38, is taken as 0.  tanh GELU the same with
    e^-2u: u = 0.798 (h + 0.0447 h^3) is off by seven roundings (two constants, four products, a sum), 7 x 2^-24 |2u| of e^-2u.  The products with the identity are
    exact."""
    import paper_2503_02495_b200 as uoe
    h = torch.cat([torch.linspace(-95, 30, 240), torch.linspace(-1, 1, 16)]).view(64, 1, 4)
    prob = uoe.Problem(B=64, L=1, L_valid=1, d=4, n=1, k=1, m=1, c=1, d_e=4, act=act, gate=False, residual=False, dtype="f32")
    eye = torch.eye(4, device="cuda").view(1, 4, 4)
    got = uoe.uoe_mlp_tokens(prob, h.cuda(), torch.zeros(4, 1, device="cuda"), eye, eye.clone()).cpu().double()
    x = h.double()
    u2 = x if act == "silu" else 2 * (2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3)
    ref = x / (1 + torch.exp(-u2))
    rel = 3 * 2.0 ** -23 + (7 * 2.0 ** -24 * u2.abs() if act != "silu" else 0)
    diff = (got - ref).abs()
    assert (diff <= rel * ref.abs() + 2.7e-37).all(), float((diff / (rel * ref.abs() + 2.7e-37)).max())


@pytest.mark.parametrize("weights", ["bf16", "f32"])
@pytest.mark.parametrize("layer", ["W1", "W2"])
@pytest.mark.parametrize("d, d_e", [(64, 40), (136, 72), (320, 264)])
def test_an_infinite_weight_in_the_last_row_is_an_infinity(weights, layer, d, d_e):
    """No step of the contraction past the matrix may meet it: 0 * Inf would make a NaN of it."""
    c = _case(5, d, d_e, 2, 2, weights, act="identity", gate=False)
    m = make(c)
    m[layer][:, -1, 0] = float("inf")
    got = run(c, m)[1]().cpu().double().view(5, d)
    x, W1, W2 = m["x"].double().view(5, d), m["W1"].double(), m["W2"].double()
    ref = x + sum((x @ W1[i]) @ W2[i] for i in range(2))
    assert torch.isinf(ref).any() and torch.equal(torch.isnan(ref), torch.isnan(got))
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]) and torch.isfinite(got[~inf & ~torch.isnan(ref)]).all()
