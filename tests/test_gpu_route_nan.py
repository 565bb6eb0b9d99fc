"""uoe_route where gates have no order: every sample still gets k experts and every expert its patches, nothing is written past the outputs, and
the other samples keep their bits.  (Ranked by comparisons alone, a NaN gate is beaten by none: a sample would choose all n experts and write
n - k numbers past its own.)"""
import pytest
import torch

import uoe_inputs as gen
from tests.helpers import problem_of, to_dev

pytestmark = pytest.mark.gpu

CASES = {
    "small": gen.tiny(B=3, dtype="f32"),
    "bf16": gen.tiny(B=5, L=112, L_valid=100, m=7, c=4, d=136, n=9, k=2, d_ff=9 * 72, dtype="bf16"),
    "many_samples": gen.tiny(B=70, L=64, L_valid=60, m=8, c=3, d=64, n=8, k=3, d_ff=8 * 32, dtype="bf16"),
    "wide": gen.tiny(B=2, L=1024, L_valid=1024, m=64, c=5, d=1024, n=16, k=4, d_ff=16 * 64, dtype="bf16"),
    "whole_samples": gen.tiny(B=6, L=64, L_valid=64, m=4, c=4, d=64, n=6, k=2, d_ff=6 * 32, dtype="bf16"),
    "one_token": gen.tiny(B=40, L=1, L_valid=1, m=1, c=1, d=128, n=12, k=3, d_ff=12 * 32, dtype="bf16"),
    "all_experts": gen.tiny(B=4, L=64, L_valid=64, m=8, c=3, d=64, n=4, k=4, d_ff=4 * 32, dtype="bf16"),
}


def _guarded(uoe, prob):
    """Routing outputs with 256 words behind each that nobody may touch."""
    r, guards = uoe.alloc_routing(prob), []
    for f in ("expert_idx", "patch_idx", "gate", "p_samp", "p_patch", "expert_offsets"):
        t = getattr(r, f)
        buf = torch.full((t.numel() + 256,), -77, dtype=t.dtype, device="cuda")
        setattr(r, f, buf[:t.numel()].view(t.shape))
        guards.append(buf[t.numel():])
    return r, guards


def _check_form(prob, r):
    e, p = r.expert_idx.cpu(), r.patch_idx.cpu()
    assert (e >= 0).all() and (e < prob.n).all() and (e[:, 1:] > e[:, :-1]).all()
    assert (p < prob.m).all()
    cnt = torch.bincount(e.flatten().long(), minlength=prob.n) * prob.l_a
    assert r.expert_offsets.cpu().tolist() == [0] + torch.cumsum((cnt + 127) // 128 * 128, 0).tolist()


@pytest.mark.parametrize("static", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", list(CASES))
def test_a_sample_without_an_order(name, bad, static):
    import paper_2503_02495_b200 as uoe
    w = CASES[name]
    prob = problem_of(w, "mlp")
    x, Wr = to_dev(gen.make_x(w)), to_dev(gen.store(gen.make_router(w).f64 * 20, w.dtype))
    route = (lambda x, r: uoe.uoe_route_static(prob, x, Wr, out=r)) if static else (lambda x, r: uoe.uoe_route(prob, x, Wr, out=r))
    ref, _ = _guarded(uoe, prob)
    route(x, ref)
    for b in (0, prob.B - 1):
        t = min(prob.l_p, prob.L_valid) - 1                      # a real token of patch 0
        x2 = x.clone()
        x2[b, t, 3] = bad
        r, guards = _guarded(uoe, prob)
        route(x2, r)
        torch.cuda.synchronize()
        assert all((g == -77).all() for g in guards)
        _check_form(prob, r)
        keep = torch.arange(prob.B) != b
        for f in ("expert_idx", "patch_idx", "gate", "p_samp", "p_patch"):
            assert torch.equal(getattr(r, f)[keep], getattr(ref, f)[keep]), f
        assert torch.isnan(r.p_samp[b]).all() and r.expert_idx[b].tolist() == list(range(prob.k))
        # patch 0 has no order and comes last: the c best of the others, or every patch where c takes them all
        elig = -(-prob.L_valid // prob.l_p)
        take = min(prob.c, elig)
        pp = r.p_patch[b].cpu()
        assert torch.isnan(pp[:, 0]).all()
        for s, i in enumerate(r.expert_idx[b].tolist()):
            v = torch.where(torch.isnan(pp[i]), torch.full_like(pp[i], -1), pp[i])[:elig]
            best = sorted(sorted(range(elig), key=lambda j: (-float(v[j]), j))[:take])
            assert r.patch_idx[b, s].tolist() == best + [-1] * (prob.c - take)


def test_all_gates_of_a_sample_without_an_order():
    import paper_2503_02495_b200 as uoe
    w = CASES["bf16"]
    prob = problem_of(w, "mlp")
    x, Wr = to_dev(gen.make_x(w)), to_dev(gen.make_router(w))
    x[prob.B - 1] = float("nan")
    r, guards = _guarded(uoe, prob)
    uoe.uoe_route(prob, x, Wr, out=r)
    assert all((g == -77).all() for g in guards)
    _check_form(prob, r)
    assert r.patch_idx[prob.B - 1].tolist() == [list(range(prob.c))] * prob.k
