"""rlcs_distill_loss against its definition in 64 bits, and its gradient against differences."""
import math

import pytest
import torch

import paged_plain as plain
import paper_2608_17641_amd as rl

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def inputs(M, V, K, dtype, seed, T=1.0, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((M, V), generator=g) * scale).to(dtype)
    teacher = torch.log_softmax(x.double() / T * 0.8 + torch.randn((M, V), generator=g), -1)
    top = torch.topk(teacher, min(K, V))
    ids, lp = top.indices.to(torch.int32), top.values.float()
    if K > V:
        ids = torch.cat([ids, torch.full((M, K - V), -1, dtype=torch.int32)], 1)
        lp = torch.cat([lp, torch.zeros((M, K - V))], 1)
    w = torch.rand(M, generator=g)
    w[torch.rand(M, generator=g) < 0.2] = 0.0
    return x, ids, lp, w


def check(x, ids, lp, w, T, tail, got):
    """A log-probability errs by the rounding of its logit's distance from the largest (log2 e / T of it) and of the sum; a share of
    the teacher by that of its logarithm; the class outside the list by what 1 - sum t loses."""
    loss, grad = got[0].double().cpu(), got[1].double().cpu()
    xd = x.double()
    want, want_g = plain.distill(xd, ids, lp.double(), w.double(), T, tail)
    V = x.shape[1]
    span = float((xd.amax(-1) - torch.where(xd == -math.inf, math.inf, xd).amin(-1)).max()) / T if V else 0.0
    far = float(torch.where(torch.isfinite(lp), lp, 0.0).abs().max()) if lp.numel() else 0.0
    e = EPS * (8 * (span + far) + V / 64 + 64)
    # (sum of t |log t| + t |log p| bounds what the errors of the logarithms come to)
    size = w.double() * (span + far + math.log(max(V, 2)) + 1)
    both = torch.isfinite(want)
    assert torch.equal(both, torch.isfinite(loss))
    assert bool(((loss - want).abs()[both] <= (e * (size + 1))[both] + 1e-30).all()), float((loss - want).abs()[both].max())
    # a gradient's parts are p, t and, outside the list, p t' / p'
    p = torch.nan_to_num(torch.softmax(xd / T, -1))
    parts = p + (want_g * T / w.double().clamp(min=1e-30)[:, None] - p).abs() + 1e-9
    allowed = (w.double()[:, None] / T) * parts * e * 8
    if x.dtype == torch.bfloat16:
        allowed = allowed + 2.0 ** -8 * want_g.abs() + 1e-38
    assert bool(((grad - want_g).abs() <= allowed + 1e-37).all()), float(((grad - want_g).abs() - allowed).max())


SIZES = [(1, 1, 1), (3, 5, 2), (5, 18, 18), (7, 18, 30), (40, 255, 4), (9, 1000, 64), (6, 1025, 1), (5, 3000, 200), (4, 9001, 1000), (3, 17000, 33), (2, 40001, 64),
         (2, 70007, 128), (300, 33001, 3)]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_against_definition(size, dtype, tail):
    M, V, K = SIZES[size]
    x, ids, lp, w = inputs(M, V, K, dtype, size)
    dev = [t.cuda() for t in (x, ids, lp, w)]
    got = rl.rlcs_distill_loss(*dev, tail=tail)
    check(x, ids, lp, w, 1.0, tail, got)
    assert all(torch.equal(a, b) for a, b in zip(got, rl.rlcs_distill_loss(*dev, tail=tail)))
    x, ids, lp, w = inputs(M, V, K, dtype, size + 100, T=0.6)
    dev = [t.cuda() for t in (x, ids, lp)]
    one = torch.ones(M)
    got = rl.rlcs_distill_loss(*dev, temperature=0.6, tail=tail)
    check(x, ids, lp, one, float(torch.tensor(0.6)), tail, got)
    assert torch.equal(rl.rlcs_distill_loss(*dev, temperature=0.6, tail=tail, want_grad=False)[0], got[0])
    own = dev[0].clone()
    again = rl.rlcs_distill_loss(own, *dev[1:], dlogits=own, temperature=0.6, tail=tail)
    assert again[1] is own and torch.equal(own, got[1]) and torch.equal(again[0], got[0])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [60, 700, 5000, 20000, 300001])
def test_lists(V, tail):
    """Ids listed twice, ids that are no tokens, shares of nothing, nothing listed."""
    M, K = 8, 40
    x, ids, lp, w = inputs(M, V, K, torch.float32, V)
    w[:] = 1.0
    lp = lp - 0.7  # (so that twice the mass of some is less than 1)
    ids[0, 1], ids[0, 7] = ids[0, 0], ids[0, 0]
    ids[1] = ids[1, 0]
    lp[1] = lp[1] - 4.0
    ids[2, ::2], ids[3] = -1, V
    lp[4, 3:] = -math.inf
    lp[5] = -math.inf
    ids[6, 0], ids[6, 1] = 0, V - 1
    got = rl.rlcs_distill_loss(x.cuda(), ids.cuda(), lp.cuda(), tail=tail)
    check(x, ids, lp, w, 1.0, tail, got)
    none = rl.rlcs_distill_loss(x.cuda(), ids[:, :0].cuda(), lp[:, :0].cuda(), tail=tail)
    check(x, ids[:, :0], lp[:, :0], w, 1.0, tail, none)
    assert not bool(none[0].any())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [90, 3000, 40000])
def test_masked_and_odd_logits(V, dtype, tail):
    M, K = 9, 8
    x, ids, lp, w = inputs(M, V, K, dtype, 5)
    w[:] = 1.0
    out = [j for j in range(V) if j not in ids[1].tolist()]
    x[0, ids[0, 2].item()] = -math.inf  # a listed token is masked: an infinite loss
    x[1, out] = -math.inf               # everything that is not listed is masked
    x[2] = -math.inf
    x[3, ::3] = torch.finfo(dtype).min
    x[4] = torch.finfo(dtype).min
    got = rl.rlcs_distill_loss(x.cuda(), ids.cuda(), lp.cuda(), tail=tail)
    for rows in ([0, 1], [3, 4], [5, 6, 7, 8]):
        check(x[rows], ids[rows], lp[rows], w[rows], 1.0, tail, [t.cpu()[rows] for t in got])
    assert math.isinf(float(got[0][0])) and math.isinf(float(got[0][2]))
    t = torch.softmax(lp[2].double(), 0) if not tail else torch.exp(lp[2].double())
    g = got[1][2].double().cpu()
    assert bool((g[ids[2].long()] + t).abs().max() <= 2.0 ** -7) and int((g != 0).sum()) <= K
    for bad in (math.nan, math.inf):
        y = x.clone()
        y[5, V // 2] = bad
        l2, g2 = rl.rlcs_distill_loss(y.cuda(), ids.cuda(), lp.cuda(), tail=tail)
        assert math.isnan(float(l2[5])) and bool(torch.isnan(g2[5]).all()) and torch.equal(l2[6:], got[0][6:]) and torch.equal(g2[6:], got[1][6:])
    lp2 = lp.clone()
    lp2[7, 1] = math.nan
    l2, g2 = rl.rlcs_distill_loss(x.cuda(), ids.cuda(), lp2.cuda(), tail=tail)
    assert math.isnan(float(l2[7])) and bool(torch.isnan(g2[7, ids[7, 1].item()])) and torch.equal(l2[8], got[0][8])
    w2 = w.clone()
    w2[6], w2[8] = math.nan, 0.0
    y = x.clone()
    y[8] = math.nan
    l2, g2 = rl.rlcs_distill_loss(y.cuda(), ids.cuda(), lp.cuda(), w2.cuda(), tail=tail)
    assert math.isnan(float(l2[6])) and float(l2[8]) == 0.0 and not bool(g2[8].any())


@pytest.mark.parametrize("tail", [False, True])
def test_differences(tail):
    """The gradient by central differences of the kernel's own loss: steps of 2^-6, whose third-order term is at most
    step^2 (a softmax's third derivatives are below 1), and two roundings of the loss over the step."""
    M, V, K = 4, 50, 6
    x, ids, lp, w = inputs(M, V, K, torch.float32, 8)
    w = w + 0.1
    _, g = rl.rlcs_distill_loss(x.cuda(), ids.cuda(), lp.cuda(), w.cuda(), temperature=0.8, tail=tail)
    h = 2.0 ** -6
    up = x[:, None, :] + h * torch.eye(V)
    down = x[:, None, :] - h * torch.eye(V)
    rep = lambda t: t[:, None].expand(M, V, *t.shape[1:]).contiguous().cuda()  # noqa: E731
    f = [rl.rlcs_distill_loss(y.cuda(), rep(ids), rep(lp), rep(w), temperature=0.8, tail=tail, want_grad=False)[0].double().cpu() for y in (up, down)]
    slope = (f[0] - f[1]) / (2 * h)
    bound = 2 * h * h / 0.8 ** 3 + 64 * EPS * 16 / h
    assert float((slope - g.double().cpu()).abs().max()) <= bound


def test_strides_and_autograd():
    g = torch.Generator(device="cuda").manual_seed(2)
    M, V, K = 6, 501, 5
    wide = torch.randn((M, V + 9), device="cuda", generator=g)
    x = wide[:, 3:V + 3]
    ids = torch.randint(0, V, (M, K), device="cuda", generator=g, dtype=torch.int32)
    lp = torch.log_softmax(torch.randn((M, K), device="cuda", generator=g), -1) - 0.2
    want = rl.rlcs_distill_loss(x.contiguous(), ids, lp, tail=True)
    grad = torch.zeros((M, V + 2), device="cuda")
    got = rl.rlcs_distill_loss(x, ids, lp, dlogits=grad[:, 1:V + 1], tail=True)
    assert torch.equal(got[0], want[0]) and torch.equal(grad[:, 1:V + 1], want[1]) and not bool(grad[:, 0].any()) and not bool(grad[:, -1].any())
    three = rl.rlcs_distill_loss(x.contiguous().view(2, 3, V), ids.view(2, 3, K), lp.view(2, 3, K), tail=True)
    assert three[0].shape == (2, 3) and torch.equal(three[1].view(M, V), want[1])
    w = torch.randn((7, V), device="cuda", generator=g, requires_grad=True)
    h = torch.randn((M, 7), device="cuda", generator=g)
    logits = h @ w
    loss, d = rl.rlcs_distill_loss(logits, ids, lp)
    assert not loss.requires_grad and not d.requires_grad
    logits.backward(d)
    assert torch.allclose(w.grad, h.t() @ d, rtol=1e-4, atol=1e-5)
    logits = h @ w
    later = (logits * logits).sum()
    rl.rlcs_distill_loss(logits, ids, lp, dlogits=logits.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        later.backward()


def test_no_logits():
    e = torch.empty((4, 0), device="cuda")
    loss, grad = rl.rlcs_distill_loss(e, torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda"), loss=torch.full((4,), 7.0, device="cuda"))
    assert not bool(loss.any()) and grad.shape == (4, 0)
