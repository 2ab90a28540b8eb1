"""rlcs_paged_attn where the keys are dealt out in pieces (tables of more than 1024 keys), against its definition in 64 bits: sequences
of unequal length, more of them than a wave has lanes, empty ones between them, one and two tiles of few rows, tiles of many rows beside
them, entries that are no page."""
import math
import random

import pytest
import torch

import paper_2608_17641_amd as rl
from test_gpu_paged import I32, case, check, to_gpu

pytestmark = pytest.mark.gpu


def wide(c, keys, page, holes=0.0, seed=0):
    """The case with tables of more than `keys` keys, and some entries that are no page."""
    q, k, v, table, length, start = c
    rng = random.Random(seed)
    W = max(max(len(row) for row in table), keys // page + 1)
    table = [[rng.choice([-1, -7, k.shape[0], k.shape[0] + 9]) if holes and rng.random() < holes else p for p in row] + [-1] * (W - len(row)) for row in table]
    return q, k, v, table, length, start


def mixed(B, most, chunks, seed):
    """Lengths from 0 to most, a few of them 0; chunk lengths drawn from `chunks`, no longer than their sequence."""
    rng = random.Random(seed)
    lengths = [0 if rng.random() < 0.15 else int(math.exp(rng.uniform(0, math.log(most)))) for _ in range(B)]
    lengths[rng.randrange(B)] = most
    return lengths, [min(n, rng.choice(chunks)) for n in lengths]


def run(c, scale, **kw):
    """Outputs with a row behind the last sequence, which stays as it is."""
    q, k, v, table, length, start = to_gpu(*c)
    n = q.shape[0]
    more = torch.zeros((n + 2, *q.shape[1:]), dtype=q.dtype, device="cuda")
    more[:n] = q
    o, lse = torch.full_like(more, 7.0), torch.full(more.shape[:2], 7.0, device="cuda")
    got = rl.rlcs_paged_attn(more, k, v, table, length, start, o, lse, scale=scale, **kw)
    assert bool((o[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    again = rl.rlcs_paged_attn(more, k, v, table, length, start, scale=scale, **kw)
    assert all(torch.allclose(x[:n], y[:n], rtol=0, atol=0, equal_nan=True) for x, y in zip(again, (o, lse)))
    return got[0][:n], got[1][:n]


# sequences, most keys, chunks, Hq, Hkv, D, page
FEW = [
    (150, 1500, [1], 8, 2, 64, 16),            # single tokens, four rows a tile
    (130, 1300, [1, 3, 4], 8, 2, 64, 32),      # up to sixteen rows
    (70, 1500, [1, 3, 5], 8, 2, 128, 16),      # up to twenty: two tiles
    (90, 900, [2, 4], 16, 2, 64, 64),          # sixteen and 32
    (100, 1200, [1, 2], 6, 3, 72, 16),         # dimensions that fill no tile
    (66, 700, [1, 2, 3], 8, 2, 256, 32),       # more than 128 dimensions: one tile
    (1, 9000, [1], 8, 1, 64, 16),              # one sequence in all pieces
    (3, 5000, [4, 5], 6, 1, 128, 1024),        # three, pages longer than pieces
    (40, 60, [1], 1100, 1100, 8, 16),          # more key heads than pieces
    (300, 40, [1, 2], 4, 1, 64, 16),           # pieces of several tiles
    (2, 1, [1], 2, 1, 64, 16),                 # next to nothing
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("i", range(len(FEW)))
def test_few_rows(i, dtype):
    B, most, chunks, Hq, Hkv, D, page = FEW[i]
    lengths, taken = mixed(B, most, chunks, i)
    c = wide(case(lengths, taken, Hq, Hkv, D, page, dtype, i), 1024, page)
    check(*c, 0.3, run(c, 0.3, max_chunk=max(chunks)))
    check(*c, 0.3, run(c, 0.3))  # (chunks of any length: the kernel of many rows finds none)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("i", [0, 2, 4, 7, 9])
def test_entries_that_are_no_page(i, dtype):
    B, most, chunks, Hq, Hkv, D, page = FEW[i]
    lengths, taken = mixed(B, most, chunks, i + 50)
    c = wide(case(lengths, taken, Hq, Hkv, D, page, dtype, i), 1024, page, holes=0.3, seed=i)
    check(*c, 0.3, run(c, 0.3, max_chunk=max(chunks)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,D,r,page,holes", [(100, 64, 4, 16, 0.0), (80, 128, 2, 64, 0.2), (70, 40, 8, 32, 0.0), (66, 200, 4, 16, 0.2)])
def test_many_rows_past_the_first_sequences(B, D, r, page, holes, dtype):
    """Long chunks of sequences past the 64th, single tokens and drafts before and between them."""
    lengths, taken = mixed(B, 400, [1, 2, 3], B)
    for b, (n, t) in {B - 1: (700, 150), B - 2: (130, 130), 65: (1100, 33), 30: (90, 70), B - 3: (0, 0), 64: (64, 64)}.items():
        lengths[b], taken[b] = n, t
    c = wide(case(lengths, taken, 2 * r, 2, D, page, dtype, B), 1300, page, holes, B)
    check(*c, 0.25, run(c, 0.25))
    check(*c, 0.25, run(c, 0.25, max_chunk=150))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 4, 5, 9, 40])
def test_equal_chunks(T, dtype):
    """Without q_start: every sequence has T new tokens, some of them at positions below 0."""
    lengths, _ = mixed(75, 600, [1], T)
    c = wide(case(lengths, [T] * 75, 8, 2, 64, 16, dtype, T), 1024, 16)
    dev = to_gpu(*c)
    check(*c, 0.2, rl.rlcs_paged_attn(*dev[:5], scale=0.2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,most", [(4, 3), (4, 7), (2, 40)])
def test_longer_chunks_than_said(r, most, dtype):
    """Tokens past max_chunk are left out, and left as they were."""
    lengths, taken = mixed(90, 800, [1, 2, 5, 9, 60], r + most)
    c = wide(case(lengths, taken, 2 * r, 2, 64, 16, dtype, most), 1024, 16)
    rows = torch.zeros(c[0].shape[:2], dtype=torch.bool)
    for b, n in enumerate(taken):
        rows[c[5][b]:c[5][b] + min(n, most)] = True
    q, k, v, table, length, start = to_gpu(*c)
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    got = rl.rlcs_paged_attn(q, k, v, table, length, start, o, lse, scale=0.3, max_chunk=most)
    check(*c, 0.3, got, taken=rows)
    left = (~rows).cuda()
    assert bool((o[left] == 7.0).all()) and bool((lse[left] == 7.0).all())


def test_infinite_values_in_pieces():
    """A value that is infinite or NaN shows in the tokens that see it, whichever piece it lies in."""
    lengths, taken = [1400, 900, 1, 1300] * 20, [5, 3, 1, 2] * 20
    q, k, v, table, length, start = wide(case(lengths, taken, 8, 2, 64, 16, torch.bfloat16, 4), 1024, 16)
    want = [t.cpu() for t in run((q, k, v, table, length, start), 0.3)]
    for b, pos, odd in ((0, 1398, math.inf), (41, 897, math.nan), (75, 1299, -math.inf)):
        v[table[b][pos // 16], pos % 16, 1, 9] = odd
    o, lse = (t.cpu() for t in run((q, k, v, table, length, start), 0.3))
    assert torch.equal(lse, want[1])
    hit = torch.zeros_like(o, dtype=torch.bool)
    for b, pos in ((0, 1398), (41, 897), (75, 1299)):
        first = start[b] + pos - (lengths[b] - taken[b])
        hit[max(first, start[b]):start[b + 1], 4:, 9] = True
    assert torch.equal(~torch.isfinite(o), hit) and torch.equal(o[~hit], want[0][~hit])
