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
