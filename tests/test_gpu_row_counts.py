"""The operators on rows of logits where there are enough long rows that a workgroup takes fewer waves a row:
the same rows against the definition, wherever they lie."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import test_gpu_policy
import test_gpu_sample

pytestmark = pytest.mark.gpu

# rows (sixteen waves each, eight, four), and lengths on both sides of what their registers hold
ROWS = [200, 300, 1100]
WAYS = [dict(), dict(k=1), dict(k=50), dict(k=256), dict(k=1500), dict(p=0.9), dict(p=0.999), dict(mp=0.05), dict(k=40, p=0.8, mp=0.02), dict(k=700, p=0.99)]


def spread(x, M):
    """M rows, those of x in turn."""
    return x.cuda().repeat((M + x.shape[0] - 1) // x.shape[0], *([1] * (x.dim() - 1)))[:M]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2050, 4100, 9000, 33001])
@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_sample(M, V, dtype, way):
    kw, n = WAYS[way], 7
    x, noise = test_gpu_sample.inputs(n, V, dtype, V + way, masked=0.1)
    x[3] = torch.round(x[3].float() * 2).to(dtype) / 2  # many equal logits
    x[4, V // 2:] = -math.inf
    x[5] = x[5] * 0.02  # nearly flat
    got = rl.rlcs_sample(spread(x, M), spread(noise, M), temperature=0.8, top_k=kw.get("k", 0), top_p=kw.get("p", 1.0), min_p=kw.get("mp", 0.0))
    test_gpu_sample.check(x, noise, [t[:n] for t in got], T=0.8, **kw)
    for t in got:
        whole = M // n * n
        assert bool((t[:whole].view(-1, n) == t[:n]).all()) and torch.equal(t[whole:], t[:M - whole])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2050, 9000, 33001])
@pytest.mark.parametrize("M", ROWS)
def test_sample_rows_of_their_own(M, V, dtype):
    n = 23
    x, noise = test_gpu_sample.inputs(n, V, dtype, V)
    g = torch.Generator().manual_seed(M)
    T = (0.3 + torch.rand(n, generator=g)) * (torch.rand(n, generator=g) > 0.2)
    k = (torch.randint(-1, 400, (n,), generator=g) * (torch.rand(n, generator=g) < 0.7)).to(torch.int32)
    p, mp = 0.5 + 0.6 * torch.rand(n, generator=g), 0.1 * torch.rand(n, generator=g)
    got = rl.rlcs_sample(spread(x, M), spread(noise, M), temperature=spread(T, M), top_k=spread(k, M), top_p=spread(p, M), min_p=spread(mp, M))
    test_gpu_sample.check(x, noise, [t[:n] for t in got], T=T, k=k, p=p, mp=mp)
    for t in got:
        whole = M // n * n
        assert bool((t[:whole].view(-1, n) == t[:n]).all()) and torch.equal(t[whole:], t[:M - whole])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [16390, 33001, 50001, 60000, 110000])
@pytest.mark.parametrize("M", [200, 300])
def test_policy(M, V, dtype):
    n = 7
    x, tokens, old, adv, weight = test_gpu_policy.inputs(n, V, dtype, V, masked=0.1)
    weight[0], weight[1] = 0.0, 0.5
    args = [spread(t, M) for t in (x, tokens, old, adv, weight)]
    got = rl.rlcs_policy_loss(*args, ent_coef=0.01, temperature=0.9, **test_gpu_policy.CLIP)
    test_gpu_policy.check(x, tokens, old, adv, weight, [t[:n] for t in got], 0.01, 0.9)
    logp, ent = rl.rlcs_token_logp(*args[:2], temperature=0.9)
    test_gpu_policy.check(x, tokens, old, adv, torch.ones(n), (None, None, logp[:n], ent[:n]), 0.01, 0.9)
    for t in (*got, logp, ent):
        whole = M // n * n
        assert bool((t[:whole].view(-1, n, *t.shape[1:]) == t[:n]).all()) and torch.equal(t[whole:], t[:M - whole])
    want = [t.clone() for t in got]
    over = rl.rlcs_policy_loss(*args, dlogits=args[0], ent_coef=0.01, temperature=0.9, **test_gpu_policy.CLIP)
    assert all(torch.equal(a, b) for a, b in zip(over, want))
