"""rlcs_sample on the smallest random numbers, on equal logits away from zero, and on the longest rows."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import test_gpu_sample as base

pytestmark = pytest.mark.gpu

EPS = base.EPS
# rows on 8 lanes, 64, a wave, four waves, sixteen; several workgroups without filters
VS = [18, 300, 700, 3001, 20001, 70000]
WAYS = [dict(), dict(top_k=40), dict(top_p=0.9999), dict(min_p=0.3), dict(top_k=300, top_p=0.9999), dict(top_k=2000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VS)
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_smallest_noise(V, dtype, way):
    """Numbers below 2^-126 race by their logarithm as others do: the smallest of a few wins among
    equal logits, and a logit further ahead than their distance wins over it."""
    x = torch.full((3, V), -60.0, dtype=dtype, device="cuda")
    noise = torch.ones((3, V), device="cuda")
    a, b, c = V // 5, V // 2, V - 2
    x[:, [a, b, c]] = 0.0
    noise[:, a], noise[:, b], noise[:, c] = 1e-39, 3e-42, 1e-40
    x[1, a] = 1.0          # log(1e-39 / 3e-42) = 5.8: still b
    x[2, c] = 4.0          # log(1e-40 / 3e-42) = 3.5: c
    tokens, logp = rl.rlcs_sample(x, noise, **WAYS[way])
    if way == 3:  # (min-p of 0.3 leaves c alone in the last row)
        assert float(logp[2]) == 0.0
    assert tokens.tolist() == [b, b, c]


@pytest.mark.parametrize("V", [18, 700, 20001])
def test_smallest_noise_per_row_settings(V):
    """The same with settings in tensors, for which no row is known to be without filters."""
    x = torch.zeros((2, V), device="cuda")
    noise = torch.ones((2, V), device="cuda")
    noise[:, V // 3], noise[:, V - 1] = 1e-39, 1e-40
    p = torch.tensor([1.0, 0.99999], device="cuda")
    assert rl.rlcs_sample(x, noise, top_p=p)[0].tolist()[0] == V - 1


@pytest.mark.parametrize("V", [20001, 70000, 128000])
@pytest.mark.parametrize("centre", [20.0, -300.0, 3000.0])
def test_tied_logits_away_from_zero(V, centre):
    """bfloat16 logits around a centre whose steps (0.125, 2, 16) put hundreds of them on one level: cuts among
    them go by index, however many share it."""
    g = torch.Generator().manual_seed(V)
    step = 2.0 ** (math.floor(math.log2(abs(centre))) - 7)
    x = (torch.randn(4, V, generator=g) * 2.5 * max(1.0, step)).add_(centre).to(torch.bfloat16)
    noise = torch.empty(4, V).exponential_(generator=g)
    x, noise = x.cuda(), noise.cuda()
    T = max(1.0, step) / 1.5  # levels a weight of e^-1.5 apart at most
    for kw in (dict(p=0.9), dict(p=0.5), dict(p=0.99, mp=0.01), dict(k=100), dict(k=1000), dict(k=5000, p=0.9), dict()):
        got = rl.rlcs_sample(x, noise, temperature=T, top_k=kw.get("k", 0), top_p=kw.get("p", 1.0), min_p=kw.get("mp", 0.0))
        base.check(x, noise, got, T=T, **kw)
