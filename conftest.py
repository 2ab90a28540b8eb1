"""Tests that hold a value proven wrong. They stay as they are, run, and are expected to fail; beside each the proof, and the
test that holds the right value."""
import pytest

# Row 1 masks every logit outside the list and holds p - t for the gradient. The loss there is sum t_k (log t_k - log p_k) with S = sum t_k
# below 1. It depends on the logits through log p_k = x_k - log sum_j e^{x_j} alone, so its derivative by x_j is S p_j - t_j: p_j - t_j
# adds up to 1 - S over the row, where the gradient of any function of a softmax adds up to 0.
# tests/test_gpu_distill_tail.py has the same rows with S p - t, which autograd and differences of the loss give.
WRONG = {
    f"test_gpu_distill.py::test_masked_and_odd_logits[{V}-{dtype}-True]": "p - t is not the gradient of a loss whose shares add up to S < 1: S p - t is"
    for V in (90, 3000, 40000) for dtype in ("dtype0", "dtype1")
}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG.get(item.nodeid.rsplit("/", 1)[-1])
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, strict=True, raises=AssertionError))
