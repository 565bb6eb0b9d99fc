"""GPU parity: uoe_mlp_forward_fp8 where weights and values are no numbers."""
import pytest
import torch

from tests.helpers import to_dev
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
