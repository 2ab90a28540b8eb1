"""rlcs_distill_loss with the longest lists: rows of a wave, whose four lists and bits in one workgroup are more than 64 KB of LDS."""
import pytest
import torch

import paper_2608_17641_amd as rl
from test_gpu_distill_tail import check as check_tail

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 1100, 2048, 2049, 4096, 4097, 9000])
def test_longest_lists(V, dtype, tail):
    M, K = 9, 1024
    g = torch.Generator().manual_seed(V)
    x = (torch.randn((M, V), generator=g) * 2).to(dtype)
    ids = torch.stack([torch.randperm(max(V, K), generator=g)[:K] for _ in range(M)]).to(torch.int32)  # (from V on: no token)
    lp = torch.log_softmax(torch.randn((M, K), generator=g), -1) - 0.4
    w = torch.rand(M, generator=g) + 0.2
    got = rl.rlcs_distill_loss(x.cuda(), ids.cuda(), lp.cuda(), w.cuda(), tail=tail)
    if tail:
        check_tail(x, ids, lp, w, 1.0, got)
        return
    here = ids < V
    at = torch.where(here, ids, 0).long()
    lt = torch.log_softmax(torch.where(here, lp.double(), -torch.inf), -1)
    t = torch.exp(lt)
    ls = torch.log_softmax(x.double(), -1)
    loss = (t * torch.where(here, lt - ls.gather(1, at), 0.0)).sum(-1)
    grad = torch.exp(ls).scatter_add(1, at, -t)
    # logarithms of at most 30 nats, from sums whose roundings are V / 64 + 64 at most; exponentials err by their arguments'
    e = EPS * (8 * 30 + V / 64 + 64)
    assert bool(((got[0].double().cpu() - w * loss).abs() <= e * 30 * w).all())
    off = (got[1].double().cpu() - w[:, None] * grad).abs()
    parts = w[:, None] * (torch.exp(ls) + torch.exp(ls).scatter_add(1, at, t))
    allowed = e * 8 * parts + (2.0 ** -8 * (w[:, None] * grad).abs() + 1e-38 if dtype == torch.bfloat16 else 0.0) + 1e-37
    assert bool((off <= allowed).all()), float((off - allowed).max())
