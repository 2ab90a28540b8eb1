"""rlcs_policy_loss and rlcs_token_logp where a row's other inputs are NaN, or its logits very many."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import test_gpu_policy as base

pytestmark = pytest.mark.gpu

EPS = base.EPS
# a row on four lanes, 32 lanes, one wave, four waves, eight waves, two passes
VS = [18, 200, 700, 3001, 20001, 70000]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VS)
@pytest.mark.parametrize("which", ["logp_old", "adv", "weight"])
def test_bad_inputs_of_a_token_show(V, dtype, which):
    """A NaN among a token's inputs makes its loss and gradient NaN, as the formulas do, and nothing of
    any other token; its log-probability and entropy do not depend on it."""
    x, tokens, old, adv, weight = (t.cuda() for t in base.inputs(5, V, dtype, V))
    weight = weight + 0.5
    p = dict(ent_coef=0.02, **base.CLIP)
    want = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **p)
    spoiled = dict(logp_old=old.clone(), adv=adv.clone(), weight=weight.clone())
    spoiled[which][[1, 3]] = math.nan
    for ec in (0.0, 0.02):
        p["ent_coef"] = ec
        want = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **p)
        got = rl.rlcs_policy_loss(x, tokens, spoiled["logp_old"], spoiled["adv"], spoiled["weight"], **p)
        assert bool(torch.isnan(got[0][[1, 3]]).all())
        assert bool(torch.isnan(got[1][[1, 3]]).all())
        for a, b in zip(got, want):
            assert torch.equal(a[[0, 2, 4]], b[[0, 2, 4]])
        assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    # a token left out has none of its inputs looked at
    out = weight.clone()
    out[[1, 3]] = 0.0
    if which != "weight":
        got = rl.rlcs_policy_loss(x, tokens, spoiled["logp_old"], spoiled["adv"], out, **p)
        assert not any(bool(torch.isnan(t).any()) for t in got)


@pytest.mark.parametrize("V", VS)
def test_far_behaviour_policies(V):
    """Ratios beyond float32: an advantage of 0 adds nothing, a positive one is held at the bound, a
    negative one is infinitely bad."""
    x, tokens, old, adv, _ = (t.cuda() for t in base.inputs(3, V, torch.float32, V))
    old = old * 0 - 200.0
    adv = torch.tensor([0.0, 2.0, -1.0], device="cuda")
    loss, grad, _, _ = rl.rlcs_policy_loss(x, tokens, old, adv, **base.CLIP)
    assert float(loss[0]) == 0.0 and not bool(grad[:2].any())
    assert abs(float(loss[1]) + 2 * (1 + base.CLIP["clip_high"])) <= 8 * EPS and float(loss[2]) == math.inf
