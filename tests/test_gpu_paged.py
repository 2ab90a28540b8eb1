"""rlcs_paged_attn and rlcs_paged_write against their definitions in 64 bits."""
import math

import pytest
import torch

import paged_plain as plain
import paper_2608_17641_amd as rl

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
I32 = torch.int32


def case(lengths, chunks, Hq, Hkv, D, page, dtype, seed, extra=3, spoil=True):
    """Sequences of scattered pages; what no length covers is NaN."""
    g = torch.Generator().manual_seed(seed)
    W = max(1, max((n + page - 1) // page for n in lengths) + 1)
    pages = sum((n + page - 1) // page for n in lengths) + extra
    perm, at, table = torch.randperm(pages, generator=g).tolist(), 0, []
    k, v = (torch.randn((pages, page, Hkv, D), generator=g).to(dtype) for _ in range(2))
    used = torch.zeros((pages, page), dtype=torch.bool)
    for n in lengths:
        some = (n + page - 1) // page
        row = perm[at:at + some]
        at += some
        for t in range(n):
            used[row[t // page], t % page] = True
        table.append(row + [-1] * (W - some))
    if spoil:
        k[~used] = math.nan
        v[~used] = math.nan
    q = torch.randn((sum(chunks), Hq, D), generator=g).to(dtype)
    start = [0]
    for n in chunks:
        start.append(start[-1] + n)
    return q, k, v, table, list(lengths), start


def to_gpu(q, k, v, table, length, start):
    return (q.cuda(), k.cuda(), v.cuda(), torch.tensor(table, dtype=I32).cuda().reshape(len(length), -1), torch.tensor(length, dtype=I32).cuda(),
            torch.tensor(start, dtype=I32).cuda())


def check(q, k, v, table, length, start, scale, got, taken=None):
    """Bounds: a score is a sum of D products, of at most |q| |k|; a weight errs by the score's error;
    bfloat16 rounds the weights and the output once each."""
    clean = lambda t: torch.nan_to_num(t.double(), 0.0, 0.0, 0.0)  # noqa: E731
    want_o, want_l = plain.paged_attention(q.double(), k.double(), v.double(), table, length, start, scale)
    o, lse = got[0].double().cpu(), got[1].double().cpu()
    rows = ~torch.isnan(want_l) if taken is None else taken
    D, n = q.shape[-1], max(length, default=0)
    kn = float(clean(k).norm(dim=-1).max()) if k.numel() else 0.0
    vm = float(clean(v).abs().max()) if v.numel() else 0.0
    qn = float(clean(q).norm(dim=-1).max()) if q.numel() else 0.0
    ds = (D + 8) * EPS * abs(scale) * qn * kn + EPS * 64
    allowed = torch.full_like(want_o, (2 * ds + (n / 16 + 32) * EPS) * 2 * vm)
    if q.dtype == torch.bfloat16:
        allowed = allowed + 2.0 ** -8 * vm + 2.0 ** -8 * want_o.abs()
    ok = (o - want_o).abs() <= allowed
    assert bool(ok[rows].all()), float(((o - want_o).abs() - allowed)[rows].max())
    assert torch.equal(torch.isinf(lse[rows]), torch.isinf(want_l[rows]))
    both = rows & torch.isfinite(want_l)
    if bool(both.any()):
        bound = ds * 2 + (n / 16 + 32) * EPS + EPS * float(want_l[both].abs().max()) * 4
        assert float((lse - want_l)[both].abs().max()) <= bound


CASES = [  # lengths, chunks, Hq, Hkv, D, page
    ([1], [1], 1, 1, 8, 16),
    ([0, 1, 17], [1, 1, 1], 4, 2, 64, 16),
    ([300, 5, 64, 65, 16], [1, 1, 1, 1, 1], 8, 8, 64, 16),
    ([40, 33, 3, 700], [5, 2, 3, 1], 8, 2, 128, 16),  # drafted tokens
    ([513, 129], [4, 4], 16, 1, 64, 64),  # 64 rows a key head
    ([100, 31, 257], [100, 31, 1], 6, 3, 72, 32),  # prompts, and a single token beside them
    ([700, 90], [130, 7], 8, 1, 128, 64),
    ([65, 600], [65, 300], 4, 2, 256, 16),
    ([50, 40], [20, 9], 5, 1, 136, 128),
    ([3, 5], [7, 9], 4, 2, 64, 16),  # more new tokens than tokens: the first see nothing
    ([2100], [9], 14, 2, 128, 256),
    ([1100, 0, 1400], [0, 0, 40], 2, 2, 40, 1024),
    ([4000], [1], 8, 1, 128, 16),  # one long sequence: many parts
    ([33] * 70, [1] * 70, 2, 1, 64, 32),  # more sequences than lanes
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_definition(i, dtype):
    lengths, chunks, Hq, Hkv, D, page = CASES[i]
    c = case(lengths, chunks, Hq, Hkv, D, page, dtype, i)
    dev = to_gpu(*c)
    scale = 1 / math.sqrt(D)
    got = rl.rlcs_paged_attn(*dev)
    check(*c, scale, got)
    again = rl.rlcs_paged_attn(*dev, max_chunk=max(chunks))
    check(*c, scale, again)
    assert all(torch.equal(x, y) for x, y in zip(again, rl.rlcs_paged_attn(*dev, max_chunk=max(chunks))))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_equal_chunks(T, dtype):
    """Without q_start every sequence has as many new tokens."""
    c = case([90, 64, 41], [T] * 3, 4, 2, 64, 16, dtype, T)
    dev = to_gpu(*c)
    got = rl.rlcs_paged_attn(*dev[:5], scale=0.2)
    check(*c, 0.2, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 4, 60])
def test_entries_that_are_no_page(T, dtype):
    """-1 and numbers past the cache, anywhere: their tokens are left out, also where the rest is too."""
    c = list(case([150, 80, 64, 700], [T] * 4, 4, 1, 64, 16, dtype, T, spoil=False))
    k, v, table = c[1], c[2], c[3]
    k[0], v[0] = math.nan, math.nan  # (page 0 is what could be read in their place)
    for row in table:
        for i, p in enumerate(row):
            if p == 0:
                row[i] = -7
    table[0][3], table[0][9], table[1][0], table[1][4] = 10 ** 6, -1, len(k), 2 ** 31 - 1
    table[2][:] = [-1] * len(table[2])
    for i in (0, 5, 6, 7, 8, 40):
        table[3][i] = -2 ** 31
    dev = to_gpu(*c)
    got = rl.rlcs_paged_attn(*dev)
    check(*c, 0.125, got)
    assert not bool(got[0][dev[5][2]:dev[5][3]].any())


@pytest.mark.parametrize("T", [2, 50])
def test_nan_and_infinite(T):
    """A NaN or infinity in a key, a value or a query shows in what it takes part in, and nowhere else."""
    c = case([70, 70, 70, 70], [T] * 4, 2, 2, 64, 16, torch.float32, 3, spoil=False)
    q, k, v, table, length, start = c
    at = lambda b, t: (table[b][t // 16], t % 16)  # noqa: E731
    k[at(0, 69)][0, 3] = math.nan  # the last key: seen by the last token alone
    v[at(1, 0)][1, 5] = math.nan
    q[start[2]][0, 0] = math.nan
    k[at(3, 69)][1, :] = 3e38
    o, lse = rl.rlcs_paged_attn(*to_gpu(*c))
    o, lse = o.cpu(), lse.cpu()
    bad = torch.isnan(o)
    want = torch.zeros_like(bad)
    want[start[1] - 1, 0] = True
    want[start[1]:start[2], 1, 5] = True
    want[start[2], 0] = True
    want[start[4] - 1, 1] = bad[start[4] - 1, 1]  # (an infinite score, or a huge one)
    assert torch.equal(bad, want)
    assert torch.isnan(lse[start[1] - 1, 0]) and torch.isnan(lse[start[2], 0]) and not torch.isnan(lse[start[1]:start[2]]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,r,D,page,length", [(2, 1, 64, 16, 70), (3, 4, 128, 16, 300), (6, 4, 72, 64, 1500), (30, 2, 128, 16, 300), (90, 4, 64, 128, 2000),
                                               (300, 1, 200, 16, 300), (9, 8, 256, 64, 1200)])
def test_values_that_some_do_not_see(T, r, D, page, length, dtype):
    """An infinite or NaN value shows in the tokens that see it; the others are what they are without it."""
    Hkv = 2
    c = case([length, length - 7, 5], [T, T, min(T, 5)], r * Hkv, Hkv, D, page, dtype, T + D)
    q, k, v, table, lengths, start = c
    bad = {}
    for seq, back, head, d, x in [(0, 1, 0, 0, math.nan), (0, 2, 1, D - 1, math.inf), (0, T // 2 + 1, 1, 3, -math.inf), (1, T, 0, 7, math.nan),
                                     (1, 1, 0, 5, math.inf), (1, 2, 0, 5, -math.inf), (2, 1, 1, 6, -math.inf), (0, length, 0, D - 2, math.nan)]:
        bad[seq, max(0, lengths[seq] - back), head, d] = x
    clean = v.clone()
    for (seq, t, head, d), x in bad.items():
        at = table[seq][t // page], t % page, head, d
        v[at], clean[at] = x, 0.0
    o, lse = rl.rlcs_paged_attn(*to_gpu(*c))
    want, want_lse = rl.rlcs_paged_attn(*to_gpu(q, k, clean, table, lengths, start))
    add = torch.zeros(want.shape)
    for (seq, t, head, d), x in bad.items():
        first = max(start[seq], start[seq + 1] - (lengths[seq] - t))
        add[first:start[seq + 1], head * r:(head + 1) * r, d] += x
    assert torch.equal(lse, want_lse) and not torch.isnan(want).any() and int((add != 0).sum()) > 0
    want = torch.where(add == 0, want.cpu().float(), add)
    assert torch.equal(torch.nan_to_num(o.cpu().float(), 3e38, 2e38, -2e38), torch.nan_to_num(want, 3e38, 2e38, -2e38))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layouts(dtype):
    """Heads before tokens in a page, gaps between pages and heads, strided queries and tables."""
    c = case([100, 47], [33, 2], 4, 2, 64, 16, dtype, 11)
    q, k, v, table, length, start = to_gpu(*c)
    pages = k.shape[0]
    kt = torch.full((pages, 2, 2, 20, 72), math.nan, dtype=dtype, device="cuda")
    k2, v2 = kt[:, 0, :, :16, :64].transpose(1, 2), kt[:, 1, :, 2:18, 8:72].transpose(1, 2)
    k2.copy_(k)
    v2.copy_(v)
    wide = torch.full((2, table.shape[1] + 5), -3, dtype=I32, device="cuda")
    wide[:, :table.shape[1]] = table
    q2 = torch.zeros((q.shape[0], 6, 80), dtype=dtype, device="cuda")[:, 1:5, 8:72]
    q2.copy_(q)
    want = rl.rlcs_paged_attn(q, k, v, table, length, start, max_chunk=33)
    got = rl.rlcs_paged_attn(q2, k2, v2, wide[:, :table.shape[1]], length, start, max_chunk=33)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_rows_of_no_sequence():
    """Rows in front of, behind and past max_chunk are left as they were."""
    c = case([60, 50], [3, 40], 2, 2, 64, 16, torch.float32, 5)
    q, k, v, table, length, start = c
    q = torch.cat([q.new_full((4, 2, 64), math.nan), q, q.new_full((9, 2, 64), math.nan)])
    start = [s + 4 for s in start]
    dev = to_gpu(q, k, v, table, length, start)
    o, lse = torch.full((56, 2, 64), 7.0, device="cuda"), torch.full((56, 2), 7.0, device="cuda")
    got = rl.rlcs_paged_attn(*dev, o, lse)
    assert got[0] is o and got[1] is lse
    check(q, k, v, table, length, start, 0.125, got)
    assert bool((o[:4] == 7).all()) and bool((o[47:] == 7).all()) and bool((lse[47:] == 7).all())
    o.fill_(7.0)
    rl.rlcs_paged_attn(*dev, o, lse, max_chunk=35)
    taken = torch.zeros((56, 2), dtype=torch.bool)
    taken[4:42] = True
    check(q, k, v, table, length, start, 0.125, (o, lse), taken)
    assert bool((o[42:] == 7).all())


def test_large_scores():
    c = case([90, 400], [20, 3], 4, 2, 64, 16, torch.float32, 9)
    q = c[0] * 1e4
    for scale in (3.0, -3.0, 0.0):
        got = rl.rlcs_paged_attn(*to_gpu(q, *c[1:]), scale=scale)
        check(q, *c[1:], scale, got)


@pytest.mark.parametrize("T", [1, 48])
def test_far_pages(T):
    """Pages whose elements lie past 2^32 bytes and 2^31 elements."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    pages, page, D = 80, 16384, 128
    k = torch.zeros((pages, page, 2, D), dtype=torch.bfloat16, device="cuda")  # 2^28.4 elements a cache of 2 heads
    big = torch.empty((pages, page, 2 * 8, D), dtype=torch.bfloat16, device="cuda")[:, :, 6:8]  # 5.4 GB, 2.7e9 elements
    g = torch.Generator(device="cuda").manual_seed(T)
    last = pages - 1
    k[last].normal_(generator=g)
    big[last].copy_(k[last])
    q = torch.randn((T, 4, D), device="cuda", generator=g).to(torch.bfloat16)
    length = torch.tensor([300], dtype=I32, device="cuda")
    got = rl.rlcs_paged_attn(q, big, big, torch.tensor([[last]], dtype=I32, device="cuda"), length)
    small = k[last:].contiguous()
    want = rl.rlcs_paged_attn(q, small, small, torch.tensor([[0]], dtype=I32, device="cuda"), length)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    new = torch.randn((1, 2, D), device="cuda", generator=g).to(torch.bfloat16)
    rl.rlcs_paged_write(new, new, big, big, torch.tensor([[last]], dtype=I32, device="cuda"), length)
    assert torch.equal(big[last, 299], new[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_write(dtype):
    for i, (lengths, chunks, page) in enumerate((([40, 3, 0, 129], [5, 3, 0, 129], 16), ([70, 2], [1, 7], 64), ([33] * 70, [2] * 70, 16))):
        q, k, v, table, length, start = case(lengths, chunks, 2, 2, 40 if i else 64, page, dtype, i, spoil=False)
        if i == 0:
            table[3][2], table[0][2] = -1, 10 ** 6
        n = start[-1]
        g = torch.Generator().manual_seed(i)
        kn, vn = (torch.randn((n + 4, 2, k.shape[-1]), generator=g).to(dtype) for _ in range(2))  # (four rows of no sequence)
        want_k, want_v = k.clone(), v.clone()
        plain.paged_write(kn, vn, want_k, want_v, table, length, start)
        _, kd, vd, td, ld, sd = to_gpu(q, k, v, table, length, start)
        before = kd._version
        got = rl.rlcs_paged_write(kn.cuda(), vn.cuda(), kd, vd, td, ld, sd)
        assert got[0] is kd and got[1] is vd and kd._version == before + 1
        assert torch.equal(kd.cpu(), want_k) and torch.equal(vd.cpu(), want_v)


def test_write_layouts():
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = torch.randn((6, 2, 3, 64), device="cuda", generator=g)  # [tokens, k and v, heads, D]
    store = torch.zeros((5, 2, 3, 16, 72), device="cuda")
    k, v = (store[:, i, :, :, :64].transpose(1, 2) for i in range(2))
    table, length = torch.tensor([[3, 1], [0, 4]], dtype=I32, device="cuda"), torch.tensor([18, 2], dtype=I32, device="cuda")
    rl.rlcs_paged_write(kv[:, 0], kv[:, 1], k, v, table, length)
    for i, t in enumerate((k, v)):
        assert torch.equal(t[3, 15], kv[0, i]) and torch.equal(t[1, :2], kv[1:3, i]) and torch.equal(t[0, :2], kv[4:6, i])
        assert int((t != 0).any(-1).any(-1).sum()) == 5
    assert not bool(store[..., 64:].any())
