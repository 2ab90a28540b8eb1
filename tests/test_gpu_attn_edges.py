"""rlcs_shared_prefix_attn where keys, values or queries that count are NaN."""
import math

import pytest
import torch

import paper_2608_17641_amd as rl
import test_gpu_attn as base

pytestmark = pytest.mark.gpu

# N, G, Hq, Hkv, D, P, S: in one kernel; split with four waves an item; a wave an item; waves that share a
# prefix's keys, 64, 128 and 256 rows of it; suffixes in several parts; no prefix
PATHS = [(2, 3, 8, 2, 64, 90, 40), (1, 4, 8, 2, 128, 700, 300), (128, 1, 32, 16, 64, 600, 20), (1, 20, 4, 2, 64, 700, 30),
         (1, 50, 4, 2, 128, 700, 30), (1, 130, 4, 2, 64, 1500, 30), (1, 2, 8, 2, 64, 600, 900), (2, 3, 8, 2, 128, 0, 700),
         (1, 30, 2, 1, 256, 600, 20)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", PATHS)
@pytest.mark.parametrize("where", ["q", "kp", "ks", "every key"])
def test_bad_inputs_show(shape, dtype, where):
    """A NaN in a query, or in a key within the lengths, makes the rows that meet it NaN (output and
    log-sum-exp), and no other row."""
    N, G, Hq, Hkv, D, P, S = shape
    if where == "kp" and P == 0:
        pytest.skip("no prefix")
    q, kp, vp, ks, vs, pl, sl = (t.cuda() for t in base.inputs(*shape, dtype, sum(shape), ragged=False))
    want = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    r = Hq // Hkv
    bad = torch.zeros((N, G, Hq), dtype=torch.bool, device="cuda")
    n, g, h = N - 1, G // 2, Hkv - 1
    if where == "q":
        q[n, g, h * r, D // 3] = math.nan
        bad[n, g, h * r] = True
    elif where == "kp":
        kp[n, P // 2, h, D - 1] = math.nan
        bad[n, :, h * r:] = True
    elif where == "ks":
        ks[n, g, S // 2, h, 0] = math.nan
        bad[n, g, h * r:] = True
    else:  # (no score of a row is a number)
        kp[n, :, h] = math.nan
        ks[n, :, :, h] = math.nan
        bad[n, :, h * r:] = True
    o, lse = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    assert bool(torch.isnan(o[bad]).all()) and bool(torch.isnan(lse[bad]).all())
    assert torch.equal(o[~bad], want[0][~bad]) and torch.equal(lse[~bad], want[1][~bad])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", PATHS)
def test_bad_values_show(shape, dtype):
    """A NaN in a value within the lengths: that dimension of the rows that weigh it, nothing else."""
    N, G, Hq, Hkv, D, P, S = shape
    q, kp, vp, ks, vs, pl, sl = (t.cuda() for t in base.inputs(*shape, dtype, sum(shape), ragged=False))
    want = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    r = Hq // Hkv
    bad = torch.zeros((N, G, Hq, D), dtype=torch.bool, device="cuda")
    if P:
        vp[0, P - 1, 0, D - 1] = math.nan
        bad[0, :, :r, D - 1] = True
    vs[N - 1, G - 1, S - 1, Hkv - 1, 0] = math.nan
    bad[N - 1, G - 1, (Hkv - 1) * r:, 0] = True
    o, lse = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, pl, sl)
    assert torch.equal(torch.isnan(o), bad) and torch.equal(o[~bad], want[0][~bad]) and torch.equal(lse, want[1])
