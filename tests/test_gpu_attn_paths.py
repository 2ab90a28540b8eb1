"""Every way that attention takes its keys, on caches as they lie in use, at unusual scales, and with values
that tell every key."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import test_gpu_attn as base
import test_gpu_attn_edges

pytestmark = pytest.mark.gpu

# and a wave an item with suffixes in several parts; heads that do not fill the kernel's dimensions
PATHS = test_gpu_attn_edges.PATHS + [(64, 2, 16, 16, 8, 520, 600), (1, 20, 4, 2, 40, 700, 30), (1, 50, 4, 2, 72, 700, 30),
                                     (1, 130, 4, 2, 104, 700, 30), (1, 30, 2, 1, 200, 600, 20)]

EPS = base.EPS
DTYPES = [torch.float32, torch.bfloat16]


def lengths(shape, seed):
    """Ragged ones, the longest among them, one that ends inside a block and none at all."""
    N, G, _, _, _, P, S = shape
    g = torch.Generator().manual_seed(seed)
    pl = torch.randint(max(0, P - P // 4), P + 1, (N,), generator=g, dtype=torch.int32)
    sl = torch.randint(0, S + 1, (N, G), generator=g, dtype=torch.int32)
    pl[0] = P
    sl[0, 0], sl[-1, -1] = S, max(0, S - 1)
    if G > 2:
        sl[0, 1] = 0
    return pl, sl


def case(shape, dtype, seed=None):
    seed = sum(shape) if seed is None else seed
    q, kp, vp, ks, vs, _, _ = base.inputs(*shape, dtype, seed, ragged=False)
    return [t.cuda() for t in (q, kp, vp, ks, vs, *lengths(shape, seed))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", PATHS)
def test_layouts(shape, dtype):
    """By head, with room past the heads and the tokens, keys and values in one tensor, one prompt for all
    groups: the same bits as contiguous tensors, and nothing read from the room."""
    N, G, Hq, Hkv, D, P, S = shape
    q, kp, vp, ks, vs, pl, sl = case(shape, dtype)
    want = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    by_head = [t.transpose(-3, -2).contiguous().transpose(-3, -2) for t in (kp, vp, ks, vs)]
    got = rl.rlcs_shared_prefix_attn(q.transpose(1, 2).contiguous().transpose(1, 2), *by_head, pl, sl)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    pair = torch.full((N, P + 3, 2, Hkv + 1, D + 8), math.nan, dtype=dtype, device="cuda")
    pair[:, :P, 0, :Hkv, :D], pair[:, :P, 1, :Hkv, :D] = kp, vp
    own = torch.full((N, G, S + 5, 2, Hkv, D + 24), math.nan, dtype=dtype, device="cuda")
    own[:, :, :S, 0, :, :D], own[:, :, :S, 1, :, :D] = ks, vs
    wide = torch.full((N, G + 1, Hq + 2, D + 8), math.nan, dtype=dtype, device="cuda")
    wide[:, :G, :Hq, :D] = q
    got = rl.rlcs_shared_prefix_attn(wide[:, :G, :Hq, :D], pair[:, :P, 0, :Hkv, :D], pair[:, :P, 1, :Hkv, :D],
                                     own[:, :, :S, 0, :, :D], own[:, :, :S, 1, :, :D], pl, sl)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = [t[:1].expand(N, P, Hkv, D) for t in (kp, vp)]
    got = rl.rlcs_shared_prefix_attn(q, *one, ks, vs, pl, sl)
    ref = rl.rlcs_shared_prefix_attn(q, *(t.contiguous() for t in one), ks, vs, pl, sl)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    heads = [t[..., :1, :].expand(*t.shape) for t in (kp, vp, ks, vs)]  # one key head behind all
    got = rl.rlcs_shared_prefix_attn(q, *heads, pl, sl)
    ref = rl.rlcs_shared_prefix_attn(q, *(t.contiguous() for t in heads), pl, sl)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def some(shape):
    """Groups and sequences to check: the first and last, and a few between."""
    N, G = shape[:2]
    pick = lambda n: sorted({0, 1 % n, n - 1} | set(range(0, n, max(1, n // 2))))  # noqa: E731
    return pick(N), pick(G)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", PATHS)
@pytest.mark.parametrize("scale", [3.0, -0.2, 0.0])
def test_scales(shape, dtype, scale):
    """One key far ahead of the others, the order turned round, and all keys alike."""
    q, kp, vp, ks, vs, pl, sl = case(shape, dtype, 4)
    o, lse = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl, scale=scale)
    groups, at = some(shape)
    for n in groups:
        i = torch.tensor(at)
        c = [t.cpu() for t in (q[n:n + 1, at], kp[n:n + 1], vp[n:n + 1], ks[n:n + 1, at], vs[n:n + 1, at], pl[n:n + 1], sl[n:n + 1, at])]
        for j in range(len(at)):
            c[3][0, j, int(c[6][0, j]):] = 0  # (what does not count shall not widen the bounds)
        base.check(*c, scale, (o[n:n + 1, i.cuda()], lse[n:n + 1, i.cuda()]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", PATHS)
def test_every_value_counts(shape, dtype):
    """The values of a row are 0 but at a few keys: the first and last of the prefix and the suffix, and around
    the edges of blocks and parts. Each element of the output is one such key's weight, off by the rounding
    of its score, of the weight's own and of the output, far less than the weight."""
    N, G, Hq, Hkv, D, P, S = shape
    q, kp, vp, ks, vs, pl, sl = case(shape, dtype, 6)
    q = q * 0.125  # (weights within a factor of e^2 or so of each other)
    vp.zero_()
    vs.zero_()
    groups, seqs = some(shape)
    edges = [0, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 257, 511, 512, 513]
    marks, pls, sls = {}, pl.tolist(), sl.tolist()
    for n in groups:
        at = [j for j in edges + [pls[n] - 2, pls[n] - 1] if 0 <= j < pls[n]][-(D // 2):]
        for d, j in enumerate(dict.fromkeys(at)):
            vp[n, j, :, d] = 1.0
            marks[n, d] = j
        for g in seqs:
            at = [j for j in edges + [sls[n][g] - 2, sls[n][g] - 1] if 0 <= j < sls[n][g]][-(D // 2):]
            for d, j in enumerate(dict.fromkeys(at)):
                vs[n, g, j, :, D // 2 + d] = 1.0
                marks[n, g, D // 2 + d] = j
    scale = 1 / math.sqrt(D)
    o, lse = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    r = Hq // Hkv
    for n in groups:
        for g in seqs:
            p, s = pls[n], sls[n][g]
            if p + s == 0:
                continue
            k = torch.cat([kp[n, :p], ks[n, g, :s]]).double().cpu()
            qd = q[n, g].double().cpu()
            score = torch.einsum("khd,hrd->hrk", k, qd.view(Hkv, r, D)).reshape(Hq, p + s) * scale
            w = torch.softmax(score, -1)
            # a score is a sum of D products; bfloat16 rounds the weight and the output to 8 bits, by 2^-8 at most
            ds = (D + 8) * EPS * scale * float(qd.norm(dim=-1).max()) * float(k.norm(dim=-1).max()) + 64 * EPS
            rel = 2 * ds + ((p + s) / 16 + 64) * EPS + (2.0 ** -7 + 2.0 ** -16 if dtype == torch.bfloat16 else 0.0)
            for key, j in marks.items():
                if key[0] != n or (len(key) == 3 and key[1] != g):
                    continue
                want = w[:, j if len(key) == 2 else p + j]
                got = o[n, g, :, key[-1]].double().cpu()
                assert bool(((got - want).abs() <= rel * want).all()), (n, g, key, j, got.tolist()[:4], want.tolist()[:4])


@pytest.mark.parametrize("shape", [(1, 4, 8, 2, 64, 600, 0), (1, 20, 4, 2, 64, 600, 0), (1, 50, 4, 2, 64, 600, 0), (1, 130, 4, 2, 64, 600, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_far_tokens(shape, dtype):
    """A prefix whose tokens are as far apart as they may be: a block of it spans up to 2 GB."""
    N, G, Hq, Hkv, D, P, _ = shape
    vec = 8 if dtype == torch.bfloat16 else 4
    far = (1 << 24) - vec
    q, kp, vp, _, _, pl, _ = base.inputs(*shape, dtype, 11, ragged=False)
    room = torch.empty(P * far, dtype=dtype, device="cuda")  # 20 or 40 GB
    kd = room.as_strided((1, P, Hkv, D), (0, far, D, 1))
    vd = room[far // (2 * vec) * vec:].as_strided((1, P, Hkv, D), (0, far, D, 1))
    kd.copy_(kp)
    vd.copy_(vp)
    want = rl.rlcs_shared_prefix_attn(q.cuda(), kp.cuda(), vp.cuda())
    got = rl.rlcs_shared_prefix_attn(q.cuda(), kd, vd)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del room, kd, vd
    torch.cuda.empty_cache()
