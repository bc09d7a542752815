"""Routing to a fixed number of experts where sums and scores reach their ends: group worths past
the largest float, groups and experts that only the last bits of 64 tell apart, scales up to the
largest float, weights of logits at the ends of the float range."""
import numpy as np
import pytest

from test_gpu_topk import case, check

pytestmark = pytest.mark.gpu

FLT_MAX = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_group_worths_past_the_largest_float(sigmoid):
    """Two biases of a group add up to more than any float, of either sign: such a group holds
    experts like any other, and its worth is compared as it is."""
    f = lambda a: np.array(a, np.float32)  # noqa: E731
    biases = [(16, f([-2e38] + [-3.3e38] * 3 + [-2.1e38] * 2 + [-3e38] * 2 + [-3e38] * 8)),
              (16, f([3e38, 2e38] * 2 + [2.6e38] * 4 + [3.3e38, 1.5e38] * 2 + [2e38] * 4)),
              (64, np.full(64, -FLT_MAX, np.float32)), (64, np.full(64, FLT_MAX, np.float32)),
              (64, np.where(np.arange(64) % 16 < 15, -FLT_MAX, 0.25).astype(np.float32)),
              (64, np.where(np.arange(64) < 20, 0.125, -FLT_MAX).astype(np.float32)),
              (256, np.where(np.arange(256) < 70, 0.125, -FLT_MAX).astype(np.float32))]
    for E, bias in biases:
        g = np.random.default_rng(E).standard_normal((5, E)).astype(np.float32)
        g[0] = 0.0
        g[1, E // 4:E // 2] = -np.inf                      # a group without experts
        g[2, :E // 4 - 1] = -np.inf                        # one of a single expert
        for top in (1, 2, 3):
            for top2 in (True, False):
                check(g, case(2, 4, top, bias, 1.0, sigmoid, True, top2))
