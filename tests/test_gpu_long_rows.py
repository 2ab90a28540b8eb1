"""Sums over the longest rows that the interface admits: 2^30 logits of the policy's, 2^24 of the
sampler's. Two levels of logits, so that the sums are known without adding them up."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def two_levels(V, dtype):
    """A row of 0 and -0.357 (bfloat16 of log 0.7) in turn, and its levels' weight."""
    x = torch.zeros((1, V), dtype=dtype, device="cuda")
    x[0, 1::2] = -0.357421875
    return x, math.exp(-0.357421875)


def bound(logp):
    """A chunk's up to 64 weights one after another, chunks to more bits than that, a tree over 1024
    lanes and as many steps for the weights' own exponentials and the final logarithm: 64 + 16 roundings of the
    sum, and a few of the result."""
    return 80 * EPS + 4 * EPS * abs(logp)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 1 << 22), (torch.bfloat16, 1 << 24), (torch.bfloat16, (1 << 28) + 6),
                                     (torch.float32, 1 << 30), (torch.bfloat16, 1 << 30)])
def test_log_probability_and_entropy(dtype, V):
    x, w = two_levels(V, dtype)
    z = (V // 2) * (1 + w)
    for token in (0, V - 1):
        t = torch.tensor([token], dtype=torch.int32, device="cuda")
        logp, ent = rl.rlcs_token_logp(x, t)
        want = (math.log(w) if token % 2 else 0.0) - math.log(z)
        # sum p log p over both levels
        want_ent = math.log(z) - (V // 2) * w * math.log(w) / z
        assert abs(float(logp) - want) <= bound(want), (float(logp), want)
        assert abs(float(ent) - want_ent) <= 2 * bound(want_ent), (float(ent), want_ent)


def test_gradient():
    V = 1 << 24
    x, w = two_levels(V, torch.float32)
    z = (V // 2) * (1 + w)
    t = torch.tensor([0], dtype=torch.int32, device="cuda")
    one = torch.ones(1, device="cuda")
    _, grad, _, _ = rl.rlcs_policy_loss(x, t, one * -math.log(z), one, clip_low=1.0, clip_high=math.inf)
    # rho = 1: the gradient is p_j - 1{j = a}; logp_old's own rounding moves rho by 17 * 2^-24 at most
    for j, p in ((1, w / z), (2, 1 / z), (V - 1, w / z)):
        assert abs(float(grad[0, j]) / p - 1) <= 2 * bound(math.log(z)) + 17 * EPS, (j, float(grad[0, j]), p)


# unfiltered over several workgroups, over one of sixteen waves, of eight, then min-p over sixteen; the general
# way (a top-k above 256) over sixteen
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("way", ["parts", "one", "many", "min_p", "general"])
def test_sampled_log_probability(dtype, way):
    V = 1 << 24
    x, w = two_levels(V, dtype)
    z = (V // 2) * (1 + w)
    M = 1
    if way == "many":
        if dtype == torch.float32:
            pytest.skip("17 GB of the same logits")
        M = 257
        x = x.repeat(M, 1)
    kw = dict(parts={}, one=dict(min_p=torch.zeros(1, device="cuda")), many={}, min_p=dict(min_p=0.5),
              general=dict(top_k=V - 2))[way]
    kept = z - 2 * w if way == "general" else z  # (the two of lowest index rank: the last of the lower level)
    tokens, logp = rl.rlcs_sample(x, **kw)
    assert not bool(tokens.any())
    want = -math.log(kept)
    assert float((logp.double() - want).abs().max()) <= bound(want), (logp[:1].tolist(), want)
