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


def _prepared(c, m):
    """(call(W scales poisoned for one expert or None), problem): one workspace, behind its control block full of NaN patterns."""
    import paper_2503_02495_b200 as uoe
    prob = uoe.Problem(B=c["T"], L=1, L_valid=1, d=c["d"], n=c["n"], k=c["k"], m=1, c=1, d_e=c["d_e"], act=c["act"], gate=c["gate"],
                       residual=c["residual"], dtype="f32" if c["weights"] == "f32" else "bf16")
    ws = uoe.alloc_workspace(prob, uoe.UOE_OP_MLP_TOKENS)
    dev = {q: v.cuda() if v is not None else None for q, v in m.items()}

    def call(x=None, poison=None):
        W, s = [dev["W1"].clone(), dev["W2"].clone()], [None, None]
        if c["weights"] == "fp8":
            W, s = zip(*[uoe.uoe_fp8_quantize(w, "blocks_t") for w in W])
        for w, q in zip(W, s):
            if poison is not None:
                w[poison] = float("nan") if q is None else torch.full(w[poison].shape, 0x7f, dtype=torch.uint8, device="cuda").view(w.dtype)
                if q is not None:
                    q[poison] = float("nan")
        ws[1024:].fill_(255)                            # stale hidden rows, terms and scales: all NaN
        r = uoe.alloc_routing(prob)
        y = uoe.uoe_mlp_tokens(prob, dev["x"] if x is None else x.cuda(), dev["Wr"], W[0], W[1], s1=s[0], s2=s[1], b1=dev["b1"], b2=dev["b2"], r=r, ws=ws)
        return y, r
    return call


@pytest.mark.parametrize("weights", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("T", [3, 14, 30, 60])
def test_what_nobody_chose_and_what_a_workspace_held_stay_out(weights, T):
    c = _case(T, 200, 136, 5, 2, weights, gate=True, seed=T)
    m = make(c)
    call = _prepared(c, m)
    ref, r = call()
    assert torch.isfinite(ref).all()
    for bad in range(5):
        got, r2 = call(poison=bad)
        assert torch.equal(r2.expert_idx, r.expert_idx)
        keep = (r.expert_idx != bad).all(1)
        assert torch.equal(got[keep], ref[keep])
        assert torch.isnan(got[~keep]).all()


@pytest.mark.parametrize("weights", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("T, at", [(1, 0), (7, 3), (20, 11), (33, 32), (64, 0)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_token_without_an_order_spoils_only_itself(weights, T, at, bad):
    """Its scores have no order, so it gets the first k experts; the others' bits stay."""
    c = _case(T, 136, 72, 6, 2, weights)
    m = make(c)
    call = _prepared(c, m)
    ref, r = call()
    x = m["x"].clone()
    x[at, 0, 5] = bad
    got, r2 = call(x=x)
    keep = torch.arange(T) != at
    assert torch.equal(got[keep], ref[keep]) and torch.equal(r2.expert_idx[keep], r.expert_idx[keep])
    assert torch.isnan(got[at]).all() and r2.expert_idx[at].tolist() == [0, 1]
