"""rlcs_verify_draft against its definition in 64 bits."""
import math

import pytest
import torch

import paged_plain as plain
import paper_2608_17641_amd as rl

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def inputs(B, K, V, dtype, seed, near=0.8, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    target = (torch.randn((B, K + 1, V), generator=g) * scale).to(dtype)
    draft = (target[:, :K].float() + near * torch.randn((B, K, V), generator=g)).to(dtype)
    race = torch.empty((B, K, V)).exponential_(generator=g)
    drawn = torch.argmax(draft.float() - torch.log(race), -1).to(torch.int32)
    u, noise = torch.rand((B, K), generator=g), torch.empty((B, V)).exponential_(generator=g)
    n = torch.randint(0, K + 1, (B,), generator=g, dtype=torch.int32)
    return target, draft, drawn, u, noise, n


def check(target, draft, drawn, u, noise, n, T, Td, got):
    """A decision may differ where it hangs on less than the rounding of what it compares: probabilities err by the score's
    rounding (a logit of up to x differs from the largest by up to 2 x / T times log2 e) and by the sum's."""
    tokens, count, logp = (t.cpu() for t in got)
    B, K = drawn.shape
    x = target.double()
    V = x.shape[-1]
    sure = 0
    for b in range(B):
        nb = K if n is None else max(0, min(K, int(n[b])))
        tb, db = float(T[b]) if torch.is_tensor(T) else T, float(Td[b]) if torch.is_tensor(Td) else Td
        want, lp, margin = plain.verify(x[b], None if draft is None else draft[b].double(), drawn[b], u[b].double(), noise[b].double(), nb, tb, db)
        size = [float(torch.nan_to_num(t.double(), 0.0, 0.0, 0.0).abs().max()) for t in ([x[b]] if draft is None else [x[b], draft[b]]) if t.numel()]
        top = max(s / (t if t > 0 else math.inf) for s, t in zip(size, (tb, db)))
        err = EPS * (8 * top + V / 64 + 64)
        if margin < 64 * err:  # (the residual of near probabilities errs by more than they do)
            continue
        sure += 1
        assert int(count[b]) == len(want), (b, margin)
        assert tokens[b].tolist() == want + [-1] * (K + 1 - len(want))
        for i, v in enumerate(lp):
            assert float(logp[b, i]) == v or abs(float(logp[b, i]) - v) <= err + 4 * EPS * abs(v), (b, i)
        assert not bool(logp[b, len(want):].any())
    return sure


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (1, 1, 2), (7, 3, 5), (40, 4, 18), (9, 2, 1000), (3, 8, 1025), (2, 3, 5003), (70, 5, 300), (1, 2, 33001)])
def test_against_definition(B, K, V, dtype):
    t, d, drawn, u, noise, n = inputs(B, K, V, dtype, B + K + V)
    dev = [x.cuda() for x in (t, d, drawn, u, noise, n)]
    got = rl.rlcs_verify_draft(*dev)
    assert check(t, d, drawn, u, noise, n, 1.0, 1.0, got) >= 0.9 * B - 1
    again = rl.rlcs_verify_draft(*dev)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    got = rl.rlcs_verify_draft(*dev[:5], temperature=0.7, draft_temperature=1.3)
    check(t, d, drawn, u, noise, None, 0.7, 1.3, got)
    got = rl.rlcs_verify_draft(dev[0], None, *dev[2:], temperature=2.0, want_logp=True)
    check(t, None, drawn, u, noise, n, 2.0, 2.0, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_settings_of_their_own(dtype):
    B, K, V = 30, 3, 700
    t, d, drawn, u, noise, n = inputs(B, K, V, dtype, 1)
    T = torch.rand(B) * 2
    T[::5] = 0.0
    T[1] = math.inf
    Td = torch.rand(B) + 0.3
    Td[2] = math.inf
    for b in range(0, B, 5):  # greedy sequences whose drafts are the largest logits, now and then
        drawn[b] = torch.argmax(t[b, :K].float(), -1).to(torch.int32)
    drawn[10, 1] = 3
    n[0:20:5] = K
    dev = [x.cuda() for x in (t, d, drawn, u, noise, n)]
    got = rl.rlcs_verify_draft(*dev, temperature=T.cuda(), draft_temperature=Td.cuda())
    assert check(t, d, drawn, u, noise, n, T, Td, got) >= 25
    assert got[1][0].item() == K + 1 and got[1][10].item() == 2 and not bool(got[2][0].any())
    got = rl.rlcs_verify_draft(dev[0], None, *dev[2:], temperature=0.0)
    assert check(t, None, drawn, u, noise, n, 0.0, 1.0, got) == B
    # a draft at temperature 0 has all of its mass on its largest logit
    top = torch.argmax(d.float(), -1).to(torch.int32)
    one = rl.rlcs_verify_draft(dev[0], dev[1], top.cuda(), *dev[3:], temperature=1.0, draft_temperature=0.0)
    two = rl.rlcs_verify_draft(dev[0], None, top.cuda(), *dev[3:], temperature=1.0)
    if dtype == torch.float32:  # (bfloat16 rows tie)
        assert all(torch.equal(x, y) for x, y in zip(one, two))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 6000])
def test_masked_and_odd_logits(V, dtype):
    B, K = 12, 3
    t, d, drawn, u, noise, n = inputs(B, K, V, dtype, 2)
    n[:] = K
    inf = math.inf
    t[0] = -inf                       # every row masked
    t[1, 1] = -inf                    # the second row masked
    t[2, :, ::2] = -inf               # half of the tokens
    t[3, :, 7] = math.nan             # counts as -inf
    t[4, :, 5] = inf                  # counts as the largest number: takes all
    d[5, 0] = -inf                    # the draft has nothing
    d[6, :, 1::2] = -inf
    t[7] = torch.finfo(dtype).min     # all alike
    d[7] = torch.finfo(dtype).min
    drawn[8] = torch.tensor([-1, V, 3], dtype=torch.int32)  # no tokens
    d[9] = t[9, :K]                   # the same policy: all stand
    d[10, :, drawn[10, 0]] = inf
    t[11, :, 1:] = -inf               # one token left
    drawn[11] = 0
    dev = [x.cuda() for x in (t, d, drawn, u, noise, n)]
    got = rl.rlcs_verify_draft(*dev)
    fin = torch.finfo(dtype).max
    tc, dc = (torch.where(x == inf, torch.tensor(fin, dtype=dtype), x) for x in (t, d))
    keep = [b for b in range(B) if b not in (8,)]
    pick = lambda x: x[keep]  # noqa: E731
    check(pick(tc), pick(dc), pick(drawn), pick(u), pick(noise), pick(n), 1.0, 1.0, [pick(x.cpu()) for x in got])
    tokens, count, logp = (x.cpu() for x in got)
    assert tokens[0].tolist() == [-1] * 4 and count[0] == 1 and logp[0].tolist() == [-inf, 0, 0, 0]
    assert count[8] == 1 and 0 <= tokens[8, 0] < V
    assert count[9] == K + 1 and tokens[9, :K].tolist() == drawn[9].tolist()
    assert count[11] == K + 1 and tokens[11].tolist() == [0] * 4 and not bool(logp[11].any())
    t[4, :, 5] = 0
    assert bool(torch.isfinite(logp[tokens >= 0]).all())


def test_strides_and_given_outputs():
    B, K, V = 5, 2, 501
    t, d, drawn, u, noise, n = (x.cuda() for x in inputs(B, K, V, torch.bfloat16, 4))
    want = rl.rlcs_verify_draft(t, d, drawn, u, noise, n)
    tw = torch.zeros((K + 1, B, V + 3), dtype=torch.bfloat16, device="cuda")[..., 1:V + 1].transpose(0, 1)
    dw = torch.zeros((B, K + 2, V + 1), dtype=torch.bfloat16, device="cuda")[:, 1:K + 1, :V]
    nw = torch.zeros((B, V + 7), device="cuda")[:, 3:V + 3]
    tw.copy_(t), dw.copy_(d), nw.copy_(noise)
    tokens, count, logp = torch.empty((B, K + 1), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty((B, K + 1), device="cuda")
    ws = torch.empty(rl.rlcs_workspace_size_verify(B, K, V), dtype=torch.uint8, device="cuda")
    before = tokens._version
    got = rl.rlcs_verify_draft(tw, dw, drawn, u, nw, n, tokens, count, logp, ws=ws)
    assert got[0] is tokens and got[1] is count and got[2] is logp and tokens._version == before + 1
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    assert rl.rlcs_verify_draft(t, d, drawn, u, noise, n, want_logp=False)[2] is None


def test_no_logits():
    e = torch.empty((3, 2, 0), device="cuda")
    i = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    tokens, count, logp = rl.rlcs_verify_draft(e, e[:, :1], i, torch.zeros((3, 1), device="cuda"), torch.empty((3, 0), device="cuda"))
    assert tokens.tolist() == [[-1, -1]] * 3 and count.tolist() == [1] * 3 and logp.tolist() == [[-math.inf, 0.0]] * 3


@pytest.mark.parametrize("with_draft", [False, True])
def test_tokens_are_the_targets(with_draft):
    """Whatever the draft, the tokens are distributed as the target's. 2^17 sequences of one drafted token: each of five
    tokens' counts, of n p on average, has a deviation of at most sqrt(n p (1 - p)); five of these are allowed."""
    n, V = 1 << 17, 5
    g = torch.Generator(device="cuda").manual_seed(6)
    p = torch.tensor([0.4, 0.3, 0.2, 0.09, 0.01], device="cuda")
    q = torch.tensor([0.1, 0.5, 0.05, 0.05, 0.3], device="cuda")
    target = torch.log(p).expand(n, 2, V).contiguous()
    draft = torch.log(q).expand(n, 1, V).contiguous()
    drawn = torch.multinomial(q if with_draft else torch.tensor([0.0, 0, 1, 0, 0], device="cuda"), n, True, generator=g).to(torch.int32)[:, None]
    u, noise = torch.rand((n, 1), device="cuda", generator=g), torch.empty((n, V), device="cuda").exponential_(generator=g)
    tokens, count, logp = rl.rlcs_verify_draft(target, draft if with_draft else None, drawn, u, noise)
    seen = torch.bincount(tokens[:, 0].long(), minlength=V).double().cpu()
    pd = p.double().cpu()
    assert bool(((seen - n * pd).abs() <= 5 * torch.sqrt(n * pd * (1 - pd))).all()), seen
    stood = float((count == 2).double().mean())
    want = float(torch.minimum(p, q).sum()) if with_draft else 0.2
    assert abs(stood - want) <= 5 * math.sqrt(want * (1 - want) / n)
    assert torch.allclose(logp[:, 0], torch.log(p)[tokens[:, 0].long()], atol=1e-5)
