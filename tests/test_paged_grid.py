"""Attention over a paged cache by more workgroups than one axis of a grid holds: the grid is then a multiple of 2^20, and
the workgroups past the last sequence have none."""
import subprocess

import pytest

from paper_2608_17641_amd import build as b

PROGRAM = r"""
#include "rlcs_paged.h"

#include <cstdio>
#include <cstdlib>
#include <vector>

int main(int argc, char** argv) {
    const int B = atoi(argv[1]), Hkv = atoi(argv[2]);
    const dim3 grid = rlcs::row_grid(int64_t(B) * Hkv);
    std::vector<char> seen(size_t(B) * Hkv);
    for (unsigned y = 0; y < grid.y; ++y)
        for (unsigned x = 0; x < grid.x; ++x) {
            int b = -1, hk = -1;
            if (!rlcs::whole_tile((int64_t(y) << rlcs::kGridBits) + x, B, Hkv, b, hk)) continue;
            if (b < 0 || b >= B || hk < 0 || hk >= Hkv || seen[size_t(b) * Hkv + hk]++) return 1;
        }
    for (char c : seen)
        if (!c) return 2;
    printf("%lld workgroups\n", (long long)(grid.x) * grid.y);
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("grid")
    src, out = str(at / "grid.hip"), str(at / "grid")
    with open(src, "w") as f:
        f.write(PROGRAM)
    cmd = [b.hipcc(), "--cuda-host-only", "-O1", "-std=c++17", "-Wno-unused-value", f"-I{b.INCLUDE}", f"-I{b.CSRC}", "-o", out, src]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return out


@pytest.mark.parametrize("B,Hkv", [(1, 1), (3, 7), (131072, 8), (131073, 8), (150000, 8), (1 << 20, 1), ((1 << 20) + 1, 1), (700001, 3)])
def test_every_pair_once(program, B, Hkv):
    done = subprocess.run([program, str(B), str(Hkv)], capture_output=True, text=True)
    assert done.returncode == 0, done
    assert int(done.stdout.split()[0]) >= B * Hkv


@pytest.mark.gpu
@pytest.mark.parametrize("ragged", [False, True])
def test_more_than_one_axis(ragged):
    """131073 + 40 sequences on 8 key heads: 2^21 workgroups. What lies past q, o, lse, length and q_start is made to show: lengths
    that would be taken, outputs that would be written."""
    import torch

    import paper_2608_17641_amd as rl
    B, H, D, page = 131073 + 40, 8, 8, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    k, v = normal(5, page, H, D), normal(5, page, H, D)
    past = 1 << 18
    length = torch.full((past + 1,), 9, dtype=torch.int32, device="cuda")
    length[:B] = torch.randint(0, page + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    start = torch.arange(past + 1, dtype=torch.int32, device="cuda")
    table = torch.randint(0, 5, (past, 1), device="cuda", generator=g, dtype=torch.int32)
    q = normal(past, H, D)
    o, lse = torch.full((past, H, D), 7.0, device="cuda"), torch.full((past, H), 7.0, device="cuda")
    rl.rlcs_paged_attn(q[:B], k, v, table[:B], length[:B], start[:B + 1] if ragged else None, o[:B], lse[:B], scale=1.0, max_chunk=1)
    torch.cuda.synchronize()
    assert bool((o[B:] == 7.0).all()) and bool((lse[B:] == 7.0).all())
    for at in range(0, B, 1 << 15):
        rows = slice(at, min(at + (1 << 15), B))
        keys, values = k[table[rows, 0].long()].double(), v[table[rows, 0].long()].double()
        s = (q[rows, None].double() * keys).sum(-1)
        hidden = torch.arange(page, device="cuda")[None, :, None] >= length[rows, None, None]
        s = s.masked_fill(hidden, -torch.inf)
        want_lse = torch.logsumexp(s, 1)
        want = (torch.exp(s - torch.where(want_lse == -torch.inf, 0.0, want_lse)[:, None])[..., None] * values).sum(1)
        # a score is a sum of eight products; weights, sums and the quotient err by some units in the last place of what they are
        size = float(s[s > -torch.inf].abs().max()) + float(values.abs().max())
        assert torch.equal(torch.isinf(want_lse), torch.isinf(lse[rows]))
        some = ~torch.isinf(want_lse)
        assert float((lse[rows].double() - want_lse)[some].abs().max()) <= 64 * 2.0 ** -24 * (1 + size)
        assert float((o[rows].double() - want).abs().max()) <= 64 * 2.0 ** -24 * (1 + size) ** 2
