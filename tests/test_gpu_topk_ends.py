"""Routing to a fixed number of experts where sums and scores reach their ends: group worths past
the largest float, groups and experts that only the last bits of 64 tell apart, scales up to the
largest float, weights of logits at the ends of the float range."""
import numpy as np
import pytest

import paper_2605_28283_amd as pp
from oracle import operators as op
from test_gpu_topk import STEP, case, check, dev, flags_of, route

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


def test_groups_that_only_normalised_scores_tell_apart():
    """1 + e^-37 is 1 in 64 bits, a third of it is one step above a third."""
    g = np.full((1, 256), -np.inf, np.float32)
    g[0, [0, 32, 64]] = 0.0
    g[0, [1, 33, 65]] = [-60.0, -37.0, -60.0]
    idx, _ = check(g, case(2, 8, 1, None, 1.0, False, False, True))
    assert idx.tolist() == [[32, 33]]


@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("G,top,top2", [(8, 8, False), (8, 3, True), (1, 1, False)])
def test_the_number_of_tokens_does_not_change_the_choice(biased, sigmoid, G, top, top2):
    """c's that differ by the last bits of 64: scores next to each other beside a bias of 1 (whose
    64-bit neighbours are 2^-52 apart), or groups worth nearly the same.  The rows one by one, in
    batches of a thousand and all at once get the same experts."""
    T, E, k = 20000, 256, 8
    rng = np.random.default_rng(G + 2 * sigmoid)
    g = rng.standard_normal((T, E)).astype(np.float32)
    near = np.arange(3, E, 16)
    bias = None
    if biased:
        bias = np.zeros(E, np.float32)
        bias[near] = 1.0
        g[:, near] = -(rng.random((T, len(near))) * 8e-15).astype(np.float32)
    else:
        g -= 45.0
        g[:, near[::2]] = 0.0
        g[:, near[1::2]] = -(36.0 + 2.0 * rng.random((T, len(near) // 2))).astype(np.float32)
    c = case(k, G, top, bias, 1.0, sigmoid, True, top2)
    idx, w = route(g, c)
    for t in range(0, T, 1000):
        i2, w2 = route(g[t:t + 1000], c)
        np.testing.assert_array_equal(i2, idx[t:t + 1000])
        np.testing.assert_array_equal(w2, w[t:t + 1000])
    for t in range(0, T, 4001):
        i1, _ = route(g[t:t + 1], c)
        np.testing.assert_array_equal(i1[0], idx[t])


def weight_tolerance(g, idx, c):
    """As in test_gpu_topk, 16 roundings and |x| 2^-24 of an exponent's argument x, counted where
    it shows: x = z - m of the expert itself, m its row's (renormalised: the chosen ones') largest
    logit; the terms of the sum have a mean |x| of at most log 256 < 6.  Where x < -104 the weight
    is below every float."""
    z = np.clip(np.nan_to_num(g.astype(np.float64), nan=-np.inf, posinf=FLT_MAX), -np.inf, FLT_MAX)
    zc = np.where(idx >= 0, np.take_along_axis(z, np.maximum(idx, 0).astype(np.int64), 1), -np.inf)
    m = (zc if c["renorm"] else z).max(1, keepdims=True)
    if c["sigmoid"]:
        m = np.minimum(m, 0.0) if c["renorm"] else 0.0
        zc = np.minimum(zc, 0.0)
    with np.errstate(invalid="ignore"):
        x = np.minimum(np.nan_to_num(np.abs(zc - m), nan=0.0, posinf=104.0), 104.0)
    return (22 + x) * STEP


def check_weights(g, c):
    ref_i, ref_w = op.route_topk(g, **c)
    for reps in (1, 4100 // len(g) + 1):
        idx, w = route(np.tile(g, (reps, 1)), c)
        np.testing.assert_array_equal(idx, np.tile(ref_i, (reps, 1)))
        ref = np.tile(ref_w, (reps, 1))
        tol = np.tile(weight_tolerance(g, ref_i, c), (reps, 1)) * np.abs(ref)
        # (below the smallest normal float a weight may be flushed)
        assert (np.abs(w - ref) <= tol + 1.2e-38 * max(1.0, abs(c["scale"]))).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_weights_at_the_ends_of_the_float_range(sigmoid, renorm):
    rng = np.random.default_rng(31)
    g = np.float32(FLT_MAX) * rng.uniform(-1, 1, (12, 64)).astype(np.float32)
    g[1, ::2], g[1, 1::2] = FLT_MAX, -FLT_MAX
    g[2], g[3] = -FLT_MAX, FLT_MAX
    g[4], g[4, [5, 6, 40]] = -FLT_MAX, [0.0, 1.0, -2.0]
    g[5], g[5, 9] = 0.0, FLT_MAX
    g[6] = (rng.integers(-3, 4, 64) * 1.4e-45).astype(np.float32)
    g[7], g[7, 3:7] = -np.inf, [-FLT_MAX, FLT_MAX, np.inf, np.nan]
    g[8] = rng.uniform(-120, 0, 64)
    for bias in (None, rng.uniform(-0.2, 0.2, 64).astype(np.float32)):
        for G, top in ((1, 1), (4, 2)):
            check_weights(g, case(6, G, top, bias, 1.0, sigmoid, renorm))


def scaled(sigmoid, renorm, E, scales):
    rng = np.random.default_rng(E)
    g = (rng.standard_normal((40, E)) * 2).astype(np.float32)
    g[0], g[1], g[2] = 0.0, -30.0, 30.0
    g[3], g[3, 7] = -np.inf, -0.1
    for scale in scales:
        for k in (1, 3):
            check_weights(g, case(k, 1, 1, None, scale, sigmoid, renorm))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [24, 256])
def test_large_scales(sigmoid, renorm, E):
    """No weight passes the largest float where scale does not."""
    scaled(sigmoid, renorm, E, (3.0e38, -3.0e38, 1.9e38, 1e-30))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [24, 256])
def test_scales_up_to_the_largest_float(sigmoid, renorm, E):
    scaled(sigmoid, renorm, E, (3.3e38, FLT_MAX, -FLT_MAX))


def test_gradient_takes_scales_up_to_the_largest_float():
    import torch
    g = np.random.default_rng(5).standard_normal((9, 24)).astype(np.float32)
    for sigmoid, renorm in ((False, False), (True, False), (False, True), (True, True)):
        c = case(3, 1, 1, None, FLT_MAX, sigmoid, renorm)
        idx, _ = route(g, case(3, 1, 1, None, 1.0, sigmoid, renorm))
        dw, dg = np.full((9, 3), 2.0 ** -4, np.float32), torch.zeros((9, 24), device="cuda")
        dw[:, 1] = -0.125
        pp.prunepath_route_topk_grad(dev(g), 9, 24, 3, dev(idx, np.int32), dev(dw), FLT_MAX,
                                     flags_of(c), dg)
        ref = op.route_topk_grad(g, idx, dw, FLT_MAX, sigmoid, renorm)
        assert (np.abs(dg.cpu().numpy() - ref) <= 64 * STEP * 0.125 * FLT_MAX).all()


def test_norm_takes_an_eps_up_to_the_largest_float():
    import torch
    x = torch.randn((3, 40), device="cuda")
    u, st = torch.full((3, 40), -1.0, device="cuda"), torch.zeros((3, 2), device="cuda")
    pp.prunepath_residual_layernorm(x, None, None, 3, 40, FLT_MAX, None, None, u, st,
                                    pp.PP_NORM_F32)
    rstd = 1.0 / np.sqrt(FLT_MAX)
    assert (np.abs(st[:, 1].cpu().numpy() - rstd) <= 4 * STEP * rstd).all()
    assert bool((u.abs() <= 10 * rstd).all())


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("std", [0.1, 3.0, 40.0])
def test_gradient_is_as_near_as_the_header_says(sigmoid, renorm, std):
    """100 2^-23 |scale| max |a|, however far the logits lie apart."""
    import torch
    for T, E, k in ((40, 256, 8), (9, 112, 112), (4100, 24, 3)):
        rng = np.random.default_rng(E + k)
        g = (rng.standard_normal((T, E)) * std).astype(np.float32)
        c = case(k, 1, 1, None, 1.5, sigmoid, renorm)
        idx, _ = route(g, c)
        dw = rng.standard_normal((T, k)).astype(np.float32)
        dg = torch.zeros((T, E), device="cuda")
        pp.prunepath_route_topk_grad(dev(g), T, E, k, dev(idx, np.int32), dev(dw), 1.5,
                                     flags_of(c), dg)
        ref = op.route_topk_grad(g, idx, dw, 1.5, sigmoid, renorm)
        tol = 100 * STEP * 1.5 * np.abs(dw).max(1, keepdims=True)
        assert (np.abs(dg.cpu().numpy() - ref) <= tol).all()
        check_weights(g[:40], c)
