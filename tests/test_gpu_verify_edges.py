"""rlcs_verify_draft on rows whose numbers are far apart or all alike, and how many sequences a check against the definition covers."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
from test_gpu_verify import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,K,V", [(7, 3, 5), (40, 4, 18), (9, 2, 1000), (30, 8, 1025), (20, 3, 5003), (70, 5, 300), (4, 2, 33001)])
def test_most_sequences_are_checked(B, K, V, dtype):
    """check() leaves out what hangs on a rounding: next to nothing, whatever the temperatures and without the draft's logits."""
    t, d, drawn, u, noise, n = inputs(B, K, V, dtype, B + K + V)
    dev = [x.cuda() for x in (t, d, drawn, u, noise, n)]
    assert check(t, d, drawn, u, noise, None, 0.7, 1.3, rl.rlcs_verify_draft(*dev[:5], temperature=0.7, draft_temperature=1.3)) >= 0.9 * B - 1
    assert check(t, None, drawn, u, noise, n, 2.0, 2.0, rl.rlcs_verify_draft(dev[0], None, *dev[2:], temperature=2.0)) >= 0.9 * B - 1
    assert check(t, d, drawn, u, noise, n, 1.0, 1.0, rl.rlcs_verify_draft(*dev)) >= 0.9 * B - 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 6000, 128000])
def test_lowest_numbers_alike(V, dtype):
    """Rows of the lowest number throughout are uniform: p = q, so every token stands whose u is below 1, and the last is the race's
    over the noise alone."""
    B, K = 6, 3
    _, _, drawn, u, noise, _ = inputs(B, K, V, dtype, 1)
    t = torch.full((B, K + 1, V), torch.finfo(dtype).min, dtype=dtype)
    u.clamp_(max=0.99)
    tokens, count, logp = (x.cpu() for x in rl.rlcs_verify_draft(t.cuda(), t[:, :K].cuda(), drawn.cuda(), u.cuda(), noise.cuda()))
    assert count.tolist() == [K + 1] * B and torch.equal(tokens[:, :K], drawn)
    assert torch.equal(tokens[:, K].long(), torch.argmin(noise, -1))
    # (a logarithm in base 2 errs by some units, the sum of V equal weights by V / 64 roundings at most)
    assert float((logp.double() + math.log(V)).abs().max()) <= 2.0 ** -24 * (V / 64 + 64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 6000, 128000])
def test_draft_of_infinite_logits(V, dtype):
    """The draft's +inf counts as the type's largest number: all of q is there. The token falls unless u is below its p, and is not drawn
    where it fell; of other drafted tokens, whose q is 0, each stands that the target gives anything."""
    B, K = 16, 2
    t, d, drawn, u, noise, _ = inputs(B, K, V, dtype, 3)
    hot = (drawn[:, 0].long() + 7) % V
    d[torch.arange(B), 0, hot] = math.inf
    on = torch.arange(B) % 2 == 0
    drawn[on, 0] = hot[on].to(torch.int32)
    u[on, 0] = 0.9
    p = torch.softmax(t.double(), -1)
    assert bool((p[on, 0, hot[on]] < 0.89).all())
    tokens, count, _ = (x.cpu() for x in rl.rlcs_verify_draft(t.cuda(), d.cuda(), drawn.cuda(), u.cuda(), noise.cuda()))
    # what is left of p where the drafted token fell is p without it
    left = torch.log(p[:, 0]) - torch.log(noise.double())
    left[torch.arange(B), hot] = -math.inf
    best = torch.topk(left, 2, -1)
    sure = on & (best.values[:, 0] - best.values[:, 1] > 1e-4)
    assert int(sure.sum()) >= 6
    assert count[on].tolist() == [1] * int(on.sum()) and torch.equal(tokens[sure, 0].long(), best.indices[sure, 0])
    assert bool((count[~on] >= 2).all()) and torch.equal(tokens[~on, 0], drawn[~on, 0])


def test_far_apart():
    """Logits of 10^38 beside ordinary ones: all of the mass is on the largest, however far the others lie below."""
    B, K, V = 8, 2, 500
    t, d, drawn, u, noise, _ = inputs(B, K, V, torch.float32, 5)
    big = torch.arange(B) * 11 % V
    t[torch.arange(B), :, big] = 1e38
    t[1::2, :, 20:] = torch.finfo(torch.float32).min
    t[torch.arange(B), :, big] = 1e38
    drawn[:4] = big[:4, None].to(torch.int32)
    drawn[4:] = ((big[4:, None] + 1) % V).to(torch.int32)
    tokens, count, logp = (x.cpu() for x in rl.rlcs_verify_draft(t.cuda(), d.cuda(), drawn.cuda(), u.cuda(), noise.cuda()))
    assert count.tolist() == [K + 1] * 4 + [1] * 4
    assert torch.equal(tokens[:, 0].long(), big) and not bool(logp[torch.arange(K + 1)[None] < count[:, None]].any())
