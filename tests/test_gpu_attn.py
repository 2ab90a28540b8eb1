"""rlcs_shared_prefix_attn against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import rollout_plain

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def inputs(N, G, Hq, Hkv, D, P, S, dtype, seed, ragged=True):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    q, kp, vp, ks, vs = rand(N, G, Hq, D), rand(N, P, Hkv, D), rand(N, P, Hkv, D), rand(N, G, S, Hkv, D), rand(N, G, S, Hkv, D)
    pl = torch.randint(0, P + 1, (N,), generator=g, dtype=torch.int32) if ragged else torch.full((N,), P, dtype=torch.int32)
    sl = torch.randint(0, S + 1, (N, G), generator=g, dtype=torch.int32) if ragged else torch.full((N, G), S, dtype=torch.int32)
    return q, kp, vp, ks, vs, pl, sl


def check(q, kp, vp, ks, vs, pl, sl, scale, got):
    """Bounds: a score is a sum of D products, of at most |q| |k|; a weight errs by the score's error;
    bfloat16 rounds the weights and the output once each."""
    d = [t.double().cpu() if t is not None else None for t in (q, kp, vp, ks, vs)]
    want_o, want_l = rollout_plain.attention(*d, pl.tolist(), None if ks is None else sl.tolist(), scale)
    o, lse = got[0].double().cpu(), got[1].double().cpu()
    clean = lambda t: torch.nan_to_num(t, 0.0, 0.0, 0.0)  # noqa: E731
    D, n = q.shape[-1], kp.shape[1] + (0 if ks is None else ks.shape[2])
    keys = [clean(t) for t in (d[1], d[3]) if t is not None and t.numel()]
    vals = [clean(t) for t in (d[2], d[4]) if t is not None and t.numel()]
    kn = max([float(t.norm(dim=-1).max()) for t in keys], default=0.0)
    vm = max([float(t.abs().max()) for t in vals], default=0.0)
    ds = (D + 8) * EPS * abs(scale) * float(d[0].norm(dim=-1).max()) * kn + EPS * 64
    tol = (2 * ds + (n / 16 + 32) * EPS) * 2 * vm
    allowed = torch.full_like(want_o, tol)
    if q.dtype == torch.bfloat16:
        allowed = allowed + 2.0 ** -8 * vm + 2.0 ** -8 * want_o.abs()
    assert not bool(torch.isnan(o).any())
    assert bool(((o - want_o).abs() <= allowed).all()), float(((o - want_o).abs() - allowed).max())
    assert torch.equal(torch.isinf(lse), torch.isinf(want_l))
    dl = torch.where(torch.isinf(want_l), 0.0, lse - want_l).abs()
    assert float(dl.max()) <= ds * 2 + (n / 16 + 32) * EPS + EPS * float(clean(want_l).abs().max()) * 4


def spoil(t, lengths, axis):
    """NaN past the lengths."""
    n = t.shape[axis]
    at = torch.arange(n) >= lengths[..., None].long()
    t[at] = math.nan
    return t


SHAPES = [  # N, G, Hq, Hkv, D, P, S
    (1, 1, 1, 1, 8, 1, 0), (1, 1, 1, 1, 64, 0, 1), (2, 3, 4, 2, 64, 5, 3), (1, 8, 8, 8, 64, 257, 33), (3, 2, 7, 1, 128, 64, 17),
    (1, 16, 8, 2, 128, 300, 130), (2, 5, 6, 3, 72, 65, 64), (1, 33, 4, 4, 128, 513, 20), (1, 4, 16, 2, 256, 100, 70), (1, 2, 20, 1, 136, 31, 40),
    (1, 1, 32, 8, 128, 1500, 700), (2, 40, 8, 1, 64, 1030, 9), (1, 64, 2, 1, 128, 2049, 1), (4, 1, 3, 3, 40, 16, 16), (1, 3, 64, 2, 128, 129, 257),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
def test_against_definition(shape, dtype, ragged):
    N, G, Hq, Hkv, D, P, S = shape
    q, kp, vp, ks, vs, pl, sl = inputs(*shape, dtype, sum(shape), ragged)
    scale = 1 / math.sqrt(D)
    if ragged:
        spoil(kp, pl, 1); spoil(vp, pl, 1)
        for t in (ks, vs):
            for n in range(N):
                spoil(t[n], sl[n], 1)
    dev = [t.cuda() for t in (q, kp, vp, ks, vs, pl, sl)]
    if not ragged:
        dev[5] = dev[6] = None
    got = rl.rlcs_shared_prefix_attn(*dev)
    check(q, kp, vp, ks, vs, pl, sl, scale, got)
    again = rl.rlcs_shared_prefix_attn(*dev)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


MANY = [  # enough sequences that waves take items of their own, with every way of taking the prefix's rows
    (128, 1, 32, 16, 64, 600, 20), (8, 32, 8, 8, 64, 530, 40), (4, 64, 16, 8, 72, 600, 300), (1, 260, 16, 8, 128, 700, 33),
    (2, 130, 8, 8, 128, 515, 1), (1, 2, 600, 2, 64, 1030, 17), (1, 128, 16, 16, 8, 900, 0),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", MANY)
def test_many_items(shape, dtype):
    N, G, Hq, Hkv, D, P, S = shape
    q, kp, vp, ks, vs, pl, sl = inputs(*shape, dtype, sum(shape))
    pl[0] = P
    spoil(kp, pl, 1); spoil(vp, pl, 1)
    for t in (ks, vs):
        for n in range(N):
            spoil(t[n], sl[n], 1)
    got = rl.rlcs_shared_prefix_attn(*(t.cuda() for t in (q, kp, vp, ks, vs, pl, sl)))
    # a sample of the sequences, the first and last among them
    some = sorted({0, G - 1} | set(range(0, G, max(1, G // 3))))
    groups = sorted({0, N - 1} | set(range(0, N, max(1, N // 3))))
    at = torch.tensor(some)
    for n in groups:
        check(q[n:n + 1, at], kp[n:n + 1], vp[n:n + 1], ks[n:n + 1, at], vs[n:n + 1, at], pl[n:n + 1], sl[n:n + 1, at],
              1 / math.sqrt(D), (got[0][n:n + 1, at.cuda()], got[1][n:n + 1, at.cuda()]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [3.0, -0.2, 0.0])
def test_large_scores(dtype, scale):
    """One key far ahead of the others: weights from 1 to nothing."""
    shape = (1, 5, 8, 2, 64, 400, 90)
    q, kp, vp, ks, vs, pl, sl = inputs(*shape, dtype, 4)
    got = rl.rlcs_shared_prefix_attn(*(t.cuda() for t in (q, kp, vp, ks, vs, pl, sl)), scale=scale)
    check(q, kp, vp, ks, vs, pl, sl, scale, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_suffix_and_no_prefix(dtype):
    q, kp, vp, ks, vs, pl, sl = inputs(2, 3, 8, 2, 128, 70, 50, dtype, 5)
    got = rl.rlcs_shared_prefix_attn(q.cuda(), kp.cuda(), vp.cuda(), prefix_len=pl.cuda())
    check(q, kp, vp, None, None, pl, sl, 1 / math.sqrt(128), got)
    none = torch.zeros(2, dtype=torch.int32)
    got = rl.rlcs_shared_prefix_attn(q.cuda(), kp.cuda(), vp.cuda(), ks.cuda(), vs.cuda(), none.cuda(), sl.cuda())
    check(q, kp, vp, ks, vs, none, sl, 1 / math.sqrt(128), got)
    got = rl.rlcs_shared_prefix_attn(q.cuda(), kp.cuda(), vp.cuda(), ks.cuda(), vs.cuda(), none.cuda(), torch.zeros_like(sl).cuda())
    assert not bool(got[0].any()) and bool((got[1] == -math.inf).all())
    # lengths past what there is, or below zero
    got = rl.rlcs_shared_prefix_attn(q.cuda(), kp.cuda(), vp.cuda(), ks.cuda(), vs.cuda(), (none + 1000).cuda(), torch.full_like(sl, -5).cuda())
    check(q, kp, vp, ks, vs, none + 70, torch.zeros_like(sl), 1 / math.sqrt(128), got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layouts(dtype):
    """Caches by head, with room past their tokens, in one tensor, and a broadcast prefix."""
    N, G, Hq, Hkv, D, P, S = 2, 3, 8, 2, 64, 90, 40
    q, kp, vp, ks, vs, pl, sl = inputs(N, G, Hq, Hkv, D, P, S, dtype, 8)
    c = [t.cuda() for t in (q, kp, vp, ks, vs, pl, sl)]
    want = rl.rlcs_shared_prefix_attn(*c)
    by_head = [c[0].transpose(1, 2).contiguous().transpose(1, 2)] + [t.transpose(-3, -2).contiguous().transpose(-3, -2) for t in c[1:5]]
    got = rl.rlcs_shared_prefix_attn(*by_head, *c[5:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    both = torch.full((N, P + 6, 2, Hkv, D + 16), math.nan, dtype=dtype, device="cuda")
    both[:, :P, 0, :, :D], both[:, :P, 1, :, :D] = c[1], c[2]
    got = rl.rlcs_shared_prefix_attn(c[0], both[:, :P, 0, :, :D], both[:, :P, 1, :, :D], *c[3:])
    assert torch.equal(got[0], want[0])
    one = c[1][:1].expand(N, P, Hkv, D), c[2][:1].expand(N, P, Hkv, D)
    got = rl.rlcs_shared_prefix_attn(c[0], *one, *c[3:])
    ref = rl.rlcs_shared_prefix_attn(c[0], one[0].contiguous(), one[1].contiguous(), *c[3:])
    assert torch.equal(got[0], ref[0])
    o, lse = torch.empty_like(c[0]), torch.empty((N, G, Hq), device="cuda")
    ws = torch.empty(max(16, rl.rlcs_workspace_size_attn(N, G, Hq, Hkv, D, P, S)), dtype=torch.uint8, device="cuda")
    got = rl.rlcs_shared_prefix_attn(*c, o, lse, ws=ws)
    assert got[0] is o and got[1] is lse and torch.equal(o, want[0])
    assert rl.rlcs_shared_prefix_attn(*c, want_lse=False)[1] is None


def test_far_offsets():
    """A cache of more than 2^31 elements: its last sequence is read where it lies."""
    N, G, Hq, Hkv, D, S = 1, 3, 4, 2, 128, 1 << 23
    kv = torch.zeros((1, G, S, Hkv, D), dtype=torch.bfloat16, device="cuda")  # 6.4 G elements
    g = torch.Generator().manual_seed(3)
    tail = torch.randn((1, G, 50, Hkv, D), generator=g).to(torch.bfloat16)
    short = torch.randn((1, 7, Hkv, D), generator=g).to(torch.bfloat16)
    q = torch.randn((N, G, Hq, D), generator=g).to(torch.bfloat16)
    kv[:, :, :50] = tail.cuda()
    sl = torch.tensor([[50, 3, 49]], dtype=torch.int32)
    pl = torch.tensor([7], dtype=torch.int32)
    got = rl.rlcs_shared_prefix_attn(q.cuda(), short.cuda(), short.cuda(), kv, kv, pl.cuda(), sl.cuda())
    check(q, short, short, tail, tail, pl, sl, 1 / math.sqrt(D), got)


def test_far_tokens():
    """Tokens so far apart that offsets within one sequence pass 2^31 elements."""
    N, G, Hq, Hkv, D, n, far = 1, 2, 4, 1, 64, 300, 1 << 23
    g = torch.Generator().manual_seed(4)
    k = torch.randn((1, n, 1, D), generator=g).to(torch.bfloat16)
    v = torch.randn((1, n, 1, D), generator=g).to(torch.bfloat16)
    q = torch.randn((N, G, Hq, D), generator=g).to(torch.bfloat16)
    room = torch.empty(n * far, dtype=torch.bfloat16, device="cuda")  # 5 GB
    kd = room.as_strided((1, n, 1, D), (0, far, 0, 1))
    vd = room[far // 2:].as_strided((1, n, 1, D), (0, far, 0, 1))
    kd.copy_(k)
    vd.copy_(v)
    for prefix in (True, False):
        if prefix:
            got = rl.rlcs_shared_prefix_attn(q.cuda(), kd, vd)
            check(q, k, v, None, None, torch.tensor([n]), None, 1 / math.sqrt(D), got)
        else:
            none = torch.empty((1, 0, 1, D), dtype=torch.bfloat16, device="cuda")
            got = rl.rlcs_shared_prefix_attn(q.cuda(), none, none, kd[:, None].expand(1, G, n, 1, D), vd[:, None].expand(1, G, n, 1, D))
            check(q, k, v, None, None, torch.tensor([n]), None, 1 / math.sqrt(D), got)
    with pytest.raises(rl.RlcsError, match="INVALID_ARG"):
        rl.rlcs_shared_prefix_attn(q.cuda(), room.as_strided((1, 2, 1, D), (0, 1 << 24, 0, 1)), kd[:, :2])


def test_other_stream():
    c = [t.cuda() for t in inputs(2, 16, 8, 2, 128, 500, 60, torch.bfloat16, 5)]
    want = rl.rlcs_shared_prefix_attn(*c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = rl.rlcs_shared_prefix_attn(*c)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
