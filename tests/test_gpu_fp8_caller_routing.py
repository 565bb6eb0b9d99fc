"""uoe_mlp_forward_fp8 on routing arrays that a caller builds: an expert named several times by a sample, an index out of range, pairs whose slots
are all unused.  Reference and bounds are those of test_gpu_mlp_fp8.py."""
import pytest
import torch

from tests.helpers import to_dev, to_f64
from tests.test_gpu_mlp_fp8 import _reference, _setup

pytestmark = pytest.mark.gpu

NAMES = ["by_patch", "several_tiles", "gathered_patches_of_8", "odd_widths", "any_scale", "one_token_patches"]


def _offsets(w, r):
    cnt = torch.bincount(r.expert_idx.flatten().long(), minlength=w.n) * (w.c * w.l_p)
    off = torch.nn.functional.pad(torch.cumsum((cnt + 127) // 128 * 128, 0), (1, 0))
    return off.int().contiguous()


def _check(name, change):
    import paper_2503_02495_b200 as uoe
    w, prob, x, r, (W1, s1, v1), (W2, s2, v2), b = _setup(name)
    change(w, r)
    r.expert_offsets = _offsets(w, r)
    bd = [None if q is None else to_dev(q) for q in b]
    run = lambda **kw: uoe.uoe_mlp_forward_fp8(prob, to_dev(x), W1, s1, W2, s2, r, b1=bd[0], b2=bd[1], **kw)
    got = run()
    y, bound = _reference(w, prob, x, r, v1, v2, b)
    diff = (torch.from_numpy(to_f64(got)).view(y.shape) - y).abs()
    real = torch.arange(w.L).repeat(w.B) < w.L_valid
    assert (diff[real] <= bound[real]).all(), float((diff / bound)[real].max())
    return uoe, run, got, r


@pytest.mark.parametrize("name", NAMES)
def test_an_expert_named_several_times_adds_every_contribution(name):
    """More pairs name an expert than there are samples."""
    def change(w, r):
        r.expert_idx.fill_(w.n - 1)
        r.patch_idx.copy_(r.patch_idx[:, :1].expand_as(r.patch_idx).clone())
        r.gate.copy_(r.gate[:, :1].expand_as(r.gate).clone())
    _check(name, change)


@pytest.mark.parametrize("name", NAMES)
def test_pairs_without_a_patch(name):
    def change(w, r):
        r.patch_idx.view(w.B * w.k, w.c)[::3] = -1
        r.gate.view(w.B * w.k, w.c)[::3] = 0
    _check(name, change)


@pytest.mark.parametrize("bad", [-1, 1 << 20])
@pytest.mark.parametrize("name", NAMES)
def test_an_expert_out_of_range_is_reported(name, bad):
    """The call returns the status; samples in front of the bad one are what they are without it."""
    uoe, run, good, r = _check(name, lambda w, r: None)
    r.expert_idx[-1, 0] = bad
    y = torch.zeros_like(good)
    with pytest.raises(uoe.UoeError) as ei:
        run(y=y)
    assert ei.value.status == 6
    assert torch.equal(y[:-1], good[:-1])
