"""The library holds the policy kernels that some row length takes, and no others."""
import re

import pytest

from paper_2608_17641_amd import build as b

# type -> (kernel, its lanes or waves a row, logits or vectors a lane), one for each range of lengths
SHORT = {("small", 4, 2), ("small", 4, 4), ("small", 4, 6), ("small", 8, 8), ("small", 16, 8), ("small", 32, 8)}
REACHED = {
    "f32": SHORT | {("small", 8, 4), ("small", 64, 8), ("small", 64, 16), ("vec", 1, 8), ("vec", 4, 4), ("vec", 4, 8), ("vec", 8, 8),
                    ("rows", 8, 0), ("rows", 16, 0)},
    "bf16": SHORT | {("small", 4, 8), ("vec", 1, 1), ("vec", 1, 2), ("vec", 1, 4), ("vec", 1, 8), ("vec", 4, 4), ("vec", 4, 8), ("vec", 8, 8),
                     ("rows", 8, 0), ("rows", 16, 0)},
}


@pytest.mark.parametrize("dtype,mark", [("f32", "f"), ("bf16", "NS_6bf16_tE")])
def test_instantiations(dtype, mark):
    b.build(force=False)
    with open(b.LIB, "rb") as f:
        data = f.read()
    for loss in (0, 1):
        pattern = rf"_ZN4rlcs\d+policy_(small|vec|rows)_kernelI{mark}Lb{loss}ELi(\d+)E(?:Li(\d+)E)?EEvNS_10PolicyArgsE"
        found = {(k.decode(), int(x), int(y or 0)) for k, x, y in re.findall(pattern.encode(), data)}
        assert found == REACHED[dtype]
