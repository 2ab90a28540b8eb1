"""rlcs_token_logp and rlcs_policy_loss against the formulas in 64 bits, and the gradient against
differences of the loss."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import rollout_plain

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
CLIP = dict(clip_low=0.2, clip_high=0.28)


def inputs(M, V, dtype, seed, scale=2.5, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(M, V, generator=g) * scale).to(dtype)
    if masked:
        x[torch.rand(M, V, generator=g) < masked] = -math.inf
    tokens = torch.randint(0, V, (M,), generator=g, dtype=torch.int32)
    x[torch.arange(M), tokens.long()] = (torch.randn(M, generator=g) * scale + scale).to(dtype)
    lp = torch.log_softmax(x.double(), -1)[torch.arange(M), tokens.long()]
    old = (lp + 0.3 * torch.randn(M, generator=g, dtype=torch.float64)).float()
    adv = torch.randn(M, generator=g)
    weight = torch.rand(M, generator=g) * (torch.rand(M, generator=g) < 0.7)
    return x, tokens, old, adv, weight


def check(x, tokens, old, adv, weight, got, ent_coef, temperature):
    """Bounds: a sum of V float32 terms over at least 64 lanes, a logarithm and an exponential of a
    number of the size of the row's scaled logits, each rounded a few times."""
    want = rollout_plain.policy(x.double().cpu(), tokens.cpu(), old.cpu().double(), adv.cpu().double(), weight.cpu().double(),
                                CLIP["clip_low"], CLIP["clip_high"], ent_coef, temperature)
    y = x.double().cpu() / temperature
    fin = torch.where(y.abs() > 1e30, 0.0, y)  # (masked, or so low that it is)
    size = float(fin.abs().max())
    tol = EPS * (x.shape[1] / 64 + 16 * (2 + size))
    loss, grad, logp, ent = (None if t is None else t.double().cpu() for t in got)
    span = 2 + 2 * min(size, 104.0)
    if logp is not None:
        assert torch.equal(torch.isinf(logp), torch.isinf(want[2]))
        d = torch.where(torch.isinf(want[2]), 0.0, logp - want[2])
        assert float(d.abs().max()) <= tol, ("logp", float(d.abs().max()), tol)
    assert float((ent - want[3]).abs().max()) <= tol * span
    if loss is None:
        return
    w = weight.cpu().double()
    rho = torch.exp((want[2] - old.cpu().double()).clamp(max=20))
    rowscale = w * (adv.cpu().double().abs() * (1 + rho) + abs(ent_coef) * span)
    bad = (loss - want[0]).abs() - 4 * tol * rowscale
    assert float(bad.max()) <= 1e-12
    if grad is not None:
        rounding = 2.0 ** -8 * want[1].abs() if x.dtype == torch.bfloat16 else 0.0
        bad = (grad - want[1]).abs() - (4 * tol * rowscale[:, None] / temperature + rounding)
        assert float(bad.max()) <= 1e-12, float(bad.max())


SIZES = [(1, 1), (5, 2), (300, 18), (33, 63), (20, 64), (17, 65), (40, 127), (9, 500), (8, 1000), (7, 1024), (6, 1027), (5, 2048),
         (5, 2049), (4, 4100), (3, 8192), (3, 8200), (3, 16387), (2, 32000), (2, 33001), (2, 50001), (2, 65536), (2, 66000), (2, 131072),
         (1, 140001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,V", SIZES)
def test_against_formula(M, V, dtype):
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(M, V, dtype, M + V))
    got = rl.rlcs_policy_loss(x, tokens, old, adv, weight, ent_coef=0.01, temperature=0.9, **CLIP)
    check(x, tokens, old, adv, weight, got, 0.01, 0.9)
    logp, ent = rl.rlcs_token_logp(x, tokens, temperature=0.9)
    check(x, tokens, old, adv, torch.ones_like(weight), (None, None, logp, ent), 0.01, 0.9)
    # the same row alone gives the same bits, and so does the call again
    again = rl.rlcs_policy_loss(x, tokens, old, adv, weight, ent_coef=0.01, temperature=0.9, **CLIP)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,V", [(50, 18), (9, 500), (5, 3001), (3, 40003)])
def test_masked_logits_and_tokens(M, V, dtype):
    x, tokens, old, adv, weight = inputs(M, V, dtype, V, masked=0.5)
    tokens[0], weight[0] = -100, 1.0  # outside: left out
    tokens[1], weight[1] = V, 1.0
    weight[2] = 0.0
    x[2] = math.nan  # not looked at
    x[0] = math.nan
    if M > 3:
        x[3], weight[3], old[3] = -math.inf, 1.0, -1.0  # nothing to choose from
        adv[3] = 1.0
    if M > 4:
        x[4, tokens[4].long()], weight[4], old[4] = -math.inf, 1.0, -1.0  # the taken one is masked
        if V > 1:
            x[4, (int(tokens[4]) + 1) % V] = 0.0
    if M > 8:
        x[7], weight[7] = torch.finfo(dtype).min, 1.0  # the type's lowest value everywhere is no mask
        x[8], weight[8] = torch.finfo(dtype).min, 1.0
        x[8, tokens[8].long()] = 1.0
        old[7] = old[8] = -1.0
    x, tokens, old, adv, weight = (t.cuda() for t in (x, tokens, old, adv, weight))
    got = rl.rlcs_policy_loss(x, tokens, old, adv, weight, ent_coef=0.02, **CLIP)
    assert not any(bool(torch.isnan(t).any()) for t in got)
    xf = torch.where(torch.isnan(x.float()), 0.0, x.float()).to(dtype)
    check(xf, tokens, old, adv, weight, got, 0.02, 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 18, 511, 2048, 5001, 40000])
def test_layouts(V, dtype):
    """Rows a stride apart, at odd addresses, with the gradient over the logits, or in [N, T, V]."""
    M = 12
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(M, V, dtype, V))
    args = (tokens, old, adv, weight)
    p = dict(ent_coef=0.01, **CLIP)
    want = rl.rlcs_policy_loss(x, *args, **p)
    for pad, off in ((3, 1), (8, 0), (5, 0)):
        wide = torch.full((M, V + pad), math.nan, dtype=dtype, device="cuda")
        view = wide[:, off:off + V]
        view.copy_(x)
        check(view, *args, rl.rlcs_policy_loss(view, *args, **p), 0.01, 1.0)
        got = rl.rlcs_policy_loss(view, *args, dlogits=view, **p)  # in place
        assert got[1] is view
        check(x, *args, got, 0.01, 1.0)
        assert bool(torch.isnan(wide[:, off + V:]).all()) and bool(torch.isnan(wide[:, :off]).all())
        lp, en = rl.rlcs_token_logp(x, tokens)
        check(x, tokens, old, adv, torch.ones_like(weight), (None, None, lp, en), 0.0, 1.0)
    cube = rl.rlcs_policy_loss(x.view(3, 4, V), *(t.view(3, 4) for t in args), **p)
    assert [t.shape for t in cube] == [(3, 4), (3, 4, V), (3, 4), (3, 4)]
    assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(cube, want))
    loss, grad, logp, ent = rl.rlcs_policy_loss(x, *args, want_grad=False, **p)
    assert grad is None
    check(x, *args, (loss, None, logp, ent), 0.01, 1.0)


@pytest.mark.parametrize("V", [7, 300, 3001])
def test_gradient_against_differences(V):
    """The sum of the losses, differenced at a step of 2^-7 in a few logits: the error of a central
    difference is the third derivative's (at most about 10 weights) times h^2 / 6, and the rounding of
    the loss over h."""
    M, h = 6, 2.0 ** -7
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(M, V, torch.float32, V))
    weight = weight + 0.1
    p = dict(ent_coef=0.1, clip_low=1.0, clip_high=math.inf)  # no clip: its corner has no derivative
    _, grad, _, _ = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **p)
    for j in [0, V // 2, V - 1] + tokens.tolist()[:2]:
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        f = [rl.rlcs_policy_loss(t, tokens, old, adv, weight, want_grad=False, **p)[0].double() for t in (up, down)]
        step = (up[:, j].double() - down[:, j].double())
        num = (f[0] - f[1]) / step
        scale = weight.double() * (1 + adv.double().abs() * 4 + 0.1 * 10)
        assert bool(((num - grad[:, j].double()).abs() <= scale * (10 * h * h / 6 + 64 * EPS / h)).all())


def test_clip_boundaries():
    """Both signs of the advantage on both sides of both bounds."""
    x = torch.zeros(8, 4, device="cuda")
    tokens = torch.zeros(8, dtype=torch.int32, device="cuda")
    rho = torch.tensor([0.5, 0.9, 1.1, 2.0] * 2, dtype=torch.float64)
    old = (math.log(0.25) - torch.log(rho)).float().cuda()
    adv = torch.tensor([1.0] * 4 + [-1.0] * 4, device="cuda")
    loss, grad, _, _ = rl.rlcs_policy_loss(x, tokens, old, adv, **CLIP)
    want = torch.tensor([-0.5, -0.9, -1.1, -1.28, 0.8, 0.9, 1.1, 2.0])
    assert torch.allclose(loss.cpu(), want, atol=1e-6)
    on = torch.tensor([1, 1, 1, 0, 0, 1, 1, 1], dtype=torch.bool)
    assert torch.equal((grad.cpu() != 0).any(1), on)


def test_other_stream():
    M, V = 64, 5000
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(M, V, torch.bfloat16, 1))
    want = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **CLIP)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **CLIP)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [18, 100, 700, 3001, 20001, 70000])
def test_finite_masks(V, dtype):
    """Large negative numbers as masks: next to other logits they count as -inf, alone they weigh alike."""
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(4, V, dtype, V))
    weight = weight + 0.5
    tokens = (V - 1 - tokens % (V // 3)).to(torch.int32)
    old = old * 0 - 3.0
    hidden = x.clone()
    hidden[:, :V - V // 3] = -math.inf
    for low in (-1e4, -1e6, -1e9, -1e10, -1e30, torch.finfo(dtype).min):
        masked = torch.where(torch.isinf(hidden), torch.full_like(x, low), hidden)
        for T in (0.7, 1.0, 2.0):
            got = rl.rlcs_policy_loss(masked, tokens, old, adv, weight, ent_coef=0.02, temperature=T, **CLIP)
            check(hidden, tokens, old, adv, weight, got, 0.02, T)
            got = rl.rlcs_policy_loss(torch.full_like(x, low), tokens, old, adv, weight, ent_coef=0.02, temperature=T, **CLIP)
            check(torch.zeros_like(x), tokens, old, adv, weight, got, 0.02, T)


@pytest.mark.parametrize("V", [18, 100, 700, 3001, 20001, 70000])
def test_far_tokens(V):
    """The log-probability of a token far below the largest: its distance, to a few roundings."""
    x = torch.zeros(4, V, device="cuda")
    x[:, V // 2] = torch.tensor([1e3, 1e7, 1e10, 1e30], device="cuda")
    tokens = torch.full((4,), V - 1, dtype=torch.int32, device="cuda")
    for T in (0.7, 1.0, 3.0):
        logp, ent = rl.rlcs_token_logp(x, tokens, temperature=T)
        want = -x[:, V // 2].double() / T
        assert float((logp.double() / want - 1).abs().max()) <= 8 * EPS
        assert float(ent.abs().max()) <= 1e-12


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [18, 100, 700, 3001, 20001, 70000])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_bad_logits_show(V, dtype, bad):
    """A NaN or +inf logit makes its row's outputs NaN, as the formulas do, and no other row's."""
    x, tokens, old, adv, weight = (t.cuda() for t in inputs(5, V, dtype, V, masked=0.2))
    weight = weight + 0.5
    p = dict(ent_coef=0.02, **CLIP)
    want = rl.rlcs_policy_loss(x, tokens, old, adv, weight, **p)
    y = x.clone()
    y[1, V // 2] = bad
    y[3] = -math.inf
    y[3, V - 1] = bad
    got = rl.rlcs_policy_loss(y, tokens, old, adv, weight, **p)
    lp = rl.rlcs_token_logp(y, tokens)
    for a, b in list(zip(got, want)) + list(zip(lp, rl.rlcs_token_logp(x, tokens))):
        assert bool(torch.isnan(a[[1, 3]]).all())
        assert torch.equal(a[[0, 2, 4]], b[[0, 2, 4]])
