"""Routing to a fixed number of experts and its gradient against the plain fp64 form.

The choice is compared exactly: c is compared in 64 bits on both sides, and the random inputs hold
no two values of c that differ by rounding errors of 64 bits only.  Weights: fp32 exp of z - m,
whose argument is rounded once (|z - m| 2^-24 relative error of the result), with a few more
roundings of at most 2^-23 each: exp, 1 + exp, a quotient, a sum over at most 256 terms in a tree
(8 levels), the product with scale.  16 of them are allowed.
"""
import numpy as np
import pytest

import paper_2605_28283_amd as pp
from oracle import operators as op

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23


def flags_of(c):
    return ((pp.PP_SCORE_SIGMOID if c["sigmoid"] else 0) | (pp.PP_TOPK_RENORM if c["renorm"] else 0) |
            (pp.PP_GROUP_TOP2 if c["top2"] else 0))


def case(k=4, n_groups=1, top_groups=1, sel_bias=None, scale=1.0, sigmoid=False, renorm=False,
         top2=False):
    return dict(k=k, n_groups=n_groups, top_groups=top_groups, sel_bias=sel_bias, scale=scale,
                sigmoid=sigmoid, renorm=renorm, top2=top2)


def dev(a, dtype=np.float32):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def route(g, c, guard=7):
    """The call on buffers with `guard` values behind them, which have to stay."""
    import torch
    T, E = g.shape
    n = T * c["k"]
    idx = torch.full((n + guard,), -77, dtype=torch.int32, device="cuda")
    w = torch.full((n + guard,), -77.0, dtype=torch.float32, device="cuda")
    pp.prunepath_route_topk_logits(dev(g), T, E, c["k"], c["n_groups"], c["top_groups"],
                                   dev(c["sel_bias"]), c["scale"], flags_of(c), idx, w)
    torch.cuda.synchronize()
    idx, w = idx.cpu().numpy(), w.cpu().numpy()
    assert (idx[n:] == -77).all() and (w[n:] == -77).all()
    return idx[:n].reshape(T, -1), w[:n].reshape(T, -1)


def weight_tolerance(g, idx):
    z = np.where(np.isfinite(g), g, 0.0).astype(np.float64)
    spread = np.abs(z).max(1, keepdims=True) * 2
    return (16 + spread) * STEP


def check(g, c):
    print("route_topk T=%d E=%d %s" % (g.shape[0], g.shape[1],
                                       {k: v for k, v in c.items() if k != "sel_bias"}), flush=True)
    idx, w = route(g, c)
    ref_i, ref_w = op.route_topk(g, **c)
    np.testing.assert_array_equal(idx, ref_i)
    # below the smallest normal float a weight may be flushed
    tiny = 1.2e-38 * abs(c["scale"])
    assert (np.abs(w - ref_w) <= weight_tolerance(g, idx) * np.abs(ref_w) + tiny).all()
    assert (w[idx < 0] == 0).all()
    # the rows again and again in a long batch, which other kernels serve: the same bits
    reps = 4100 // g.shape[0] + 1
    ib, wb = route(np.tile(g, (reps, 1)), c)
    np.testing.assert_array_equal(ib, np.tile(idx, (reps, 1)))
    np.testing.assert_array_equal(wb.view(np.int32), np.tile(w.view(np.int32), (reps, 1)))
    return idx, w


def logits(T, E, seed=0, std=3.0):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((T, E)) * std).astype(np.float32)


SHAPES = [(1, 1, 1, 1, 1), (1, 2, 1, 1, 1), (7, 5, 5, 1, 1), (3, 16, 2, 1, 1), (5, 17, 17, 1, 1),
          (4, 64, 8, 8, 3), (65, 112, 8, 1, 1), (9, 112, 16, 7, 2), (33, 148, 6, 4, 4),
          (6, 160, 6, 8, 3), (130, 256, 8, 8, 4), (2, 256, 256, 1, 1), (3, 255, 40, 5, 3),
          (3, 256, 20, 16, 6), (5, 32, 30, 16, 15), (3, 253, 12, 11, 6), (2, 135, 9, 9, 9)]


@pytest.mark.parametrize("T,E,k,G,top", SHAPES)
@pytest.mark.parametrize("sigmoid", [False, True])
def test_choice_and_weights(T, E, k, G, top, sigmoid):
    g = logits(T, E, seed=E + k)
    bias = np.random.default_rng(E).standard_normal(E).astype(np.float32) * 0.1
    check(g, case(k, G, top, None, 1.0, sigmoid, True))
    check(g, case(k, G, top, bias, 2.5, sigmoid, False, top2=True))
    check(g, case(k, G, top, None, -0.5, sigmoid, False, top2=True))
    check(g, case(k, G, top, bias, 1.0, sigmoid, True))


def test_tokens_do_not_touch_each_other():
    """A token alone, and among others at any place, gets the same bits."""
    for T, c in ((513, case(8, 4, 2, logits(1, 112, 5, 0.1)[0], 1.0, True, True, True)),
                 (3001, case(8, 4, 2, logits(1, 112, 5, 0.1)[0], 1.0, True, False, True)),
                 (3001, case(9, 7, 3, None, 1.0, False, False, True)),
                 (3001, case(8, 1, 1, logits(1, 112, 5, 0.1)[0], 1.0, False, False, False))):
        g = logits(T, 112, 4)
        idx, w = route(g, c)
        for t in (0, 1, 63, 64, 300, 512, T - 1):
            i1, w1 = route(g[t:t + 1], c)
            assert (i1[0] == idx[t]).all() and w1[0].tobytes() == w[t].tobytes()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("G,top", [(1, 1), (4, 2)])
def test_equal_logits_go_to_the_lowest_index(sigmoid, G, top):
    g = np.zeros((6, 64), np.float32)
    g[1] = 3.25
    g[2] = np.tile(np.array([1, 2], np.float32), 32)
    g[3] = np.float32(np.finfo(np.float32).min)     # a mask of the lowest finite value
    g[4, 40:] = 7.0
    g[5] = -0.0
    g[5, 1::2] = 0.0
    for bias in (None, np.zeros(64, np.float32), np.full(64, 0.25, np.float32)):
        for top2 in (False, True):
            for renorm in (False, True):
                check(g, case(5, G, top, bias, 1.0, sigmoid, renorm, top2))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_masked_experts(sigmoid, biased):
    """-inf and NaN logits and biases take no part, +inf is the largest float, rows may be empty."""
    rng = np.random.default_rng(8)
    g = logits(40, 48, 9)
    g[rng.random(g.shape) < 0.5] = -np.inf
    g[rng.random(g.shape) < 0.1] = np.nan
    g[3] = -np.inf
    g[4] = np.nan
    g[5] = -np.inf
    g[5, 17] = -2.0                                  # one expert left
    g[6] = -np.inf
    g[6, 12:15] = 1.0                                # one group left
    g[7, 3] = np.inf
    g[8, :] = np.inf
    bias = None
    if biased:
        bias = rng.standard_normal(48).astype(np.float32) * 0.1
        bias[[0, 12, 30]] = -np.inf
        bias[31] = np.nan
        bias[20] = np.inf
    for G, top in ((1, 1), (4, 2), (4, 4), (16, 5)):
        for renorm in (False, True):
            for top2 in (False, True):
                idx, w = check(g, case(7, G, top, bias, 1.0, sigmoid, renorm, top2))
                assert (idx[3] == -1).all() and (idx[4] == -1).all() and np.isfinite(w).all()


@pytest.mark.parametrize("sigmoid", [False, True])
def test_scores_that_underflow_keep_renormalised_weights(sigmoid):
    """All chosen scores below the smallest float (sigmoid), or of the experts that a bias picks."""
    g = (-200.0 - 10 * np.abs(logits(9, 32, 10, 1.0))).astype(np.float32)
    bias = None
    if not sigmoid:
        g[:, 0] = 100.0
        bias = np.where(np.arange(32) < 8, -2.0, 0.0).astype(np.float32) + \
            (np.arange(32) * 1e-3).astype(np.float32)
    idx, w = check(g, case(6, 1, 1, bias, 1.0, sigmoid, True))
    assert (np.abs(w.sum(1) - 1) <= 1e-5).all()


def near_ties(T, E, seed):
    """Values of c that 32 bits cannot tell apart, and 64 bits can."""
    rng = np.random.default_rng(seed)
    steps = rng.permuted(np.tile(np.arange(E, dtype=np.int32), (T, 1)), axis=1)
    g = (np.full((T, E), 1.0, np.float32).view(np.int32) + steps).view(np.float32)
    return g, (rng.permutation(E) * 1.37e-8).astype(np.float32)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("G,top", [(1, 1), (8, 3)])
def test_near_ties_are_decided_in_64_bits(sigmoid, G, top):
    g, bias = near_ties(50, 64, 11)
    s = 1 / (1 + np.exp(-g.astype(np.float64)))
    if sigmoid:  # the case is what it says
        c32 = (s.astype(np.float32) + bias).astype(np.float32)
        assert len(np.unique(c32[0])) < 64
    for top2 in (False, True):
        check(g, case(6, G, top, bias, 1.0, sigmoid, True, top2))
        check(g, case(6, G, top, None, 1.0, sigmoid, True, top2))


def test_many_tokens_choice():
    """A long batch over random logits: every token's choice."""
    import torch
    T, E, k = 20011, 256, 8
    rng = np.random.default_rng(12)
    g = (rng.standard_normal((T, E)) * 3 * np.exp(0.5 * rng.standard_normal((T, 1)))).astype(np.float32)
    bias = (rng.standard_normal(E) * 0.05).astype(np.float32)
    s = torch.sigmoid(torch.from_numpy(g).double())
    for G, top, b in ((1, 1, bias), (8, 4, bias), (8, 3, None), (16, 5, None)):
        idx, _ = route(g, case(k, G, top, b, 1.0, True, True, True))
        c = torch.from_numpy(g).double() if b is None else s + torch.from_numpy(b).double()
        worth = (s if b is None else c).view(T, G, E // G).sort(dim=2, descending=True).values
        groups = worth[:, :, :2].sum(2).sort(dim=1, descending=True, stable=True).indices[:, :top]
        keep = torch.zeros((T, G), dtype=torch.bool).scatter_(1, groups, True)
        c = c.masked_fill(~keep.repeat_interleave(E // G, 1), -float("inf"))
        ref = c.sort(dim=1, descending=True, stable=True).indices[:, :k].int().numpy()
        np.testing.assert_array_equal(idx, ref)


@pytest.mark.parametrize("E,k,G,top", [(256, 20, 1, 1), (256, 80, 1, 1), (250, 100, 5, 3),
                                       (256, 64, 8, 4), (64, 63, 1, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_many_equal_logits(E, k, G, top, sigmoid):
    """Logits and biases of a few values each: ties in and around the cut, of experts and groups."""
    rng = np.random.default_rng(E + k)
    g = (np.round(rng.standard_normal((5, E)) * 4) / 4).astype(np.float32)
    g[3] = 0.5
    g[4, ::3] = -np.inf
    for bias in (None, np.zeros(E, np.float32), (rng.integers(0, 3, E) / 8).astype(np.float32)):
        for top2 in (False, True):
            check(g, case(k, G, top, bias, 1.0, sigmoid, True, top2))


@pytest.mark.parametrize("sigmoid", [False, True])
def test_ends_of_the_float_range(sigmoid):
    """Subnormal logits, logits near the largest floats, and biases of both kinds."""
    rng = np.random.default_rng(24)
    tiny = (rng.integers(-3, 4, (40, 64)) * 1.4e-45).astype(np.float32)
    tiny[1] = -np.abs(tiny[1]) - np.float32(1e-40)
    tiny[2] = np.float32(1.4e-45)
    huge = np.float32(np.finfo(np.float32).max) * rng.uniform(-1, 1, (40, 64)).astype(np.float32)
    huge[3, ::2], huge[3, 1::2] = np.finfo(np.float32).max, np.finfo(np.float32).min
    big = huge[5].copy()
    for g in (tiny, huge):
        for bias in (None, tiny[7], big):
            for G, top in ((1, 1), (4, 2)):
                for top2 in (False, True):
                    check(g, case(6, G, top, bias, 1.0, sigmoid, True, top2))


def test_signalling_nans_take_no_part():
    g = logits(3, 40, 23)
    bits = g.view(np.uint32)
    bits[0, 3], bits[0, 39], bits[1, :] = 0x7F800001, 0xFF812345, 0x7FA00000
    for c in (case(5), case(5, sigmoid=True, renorm=True), case(3, 4, 2, sigmoid=True, top2=True),
              case(5, sel_bias=np.full(40, 0.25, np.float32), sigmoid=True)):
        idx, _ = check(g, c)
        assert 3 not in idx[0] and 39 not in idx[0] and (idx[1] == -1).all()


def test_offsets_past_32_bits():
    """2^22 rows of 256 logits (4 GiB): the last rows as in a call of their own, forward and back."""
    import torch
    T, E, k, n = 1 << 22, 256, 2, 5
    g = torch.randn((T, E), device="cuda")
    idx, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
    dw, dg = torch.randn((T, k), device="cuda"), torch.empty((T, E), device="cuda")
    fl = pp.PP_SCORE_SIGMOID | pp.PP_TOPK_RENORM
    pp.prunepath_route_topk_logits(g, T, E, k, 1, 1, None, 1.0, fl, idx, w)
    pp.prunepath_route_topk_grad(g, T, E, k, idx, dw, 1.0, fl, dg)
    tail = [a[-n:].clone() for a in (g, idx, w, dw, dg)]
    i2, w2, d2 = torch.zeros_like(tail[1]), torch.zeros_like(tail[2]), torch.zeros_like(tail[4])
    pp.prunepath_route_topk_logits(tail[0], n, E, k, 1, 1, None, 1.0, fl, i2, w2)
    pp.prunepath_route_topk_grad(tail[0], n, E, k, i2, tail[3], 1.0, fl, d2)
    assert torch.equal(i2, tail[1]) and torch.equal(w2, tail[2]) and torch.equal(d2, tail[4])


# ------------------------------------------------------------------ gradient

def grad(g, idx, dw, c, add=None):
    import torch
    T, E = g.shape
    dg = dev(add) if add is not None else torch.full((T, E), float("nan"), device="cuda")
    dg = torch.cat([dg.reshape(-1), torch.full((5,), -77.0, device="cuda")])
    flags = flags_of(c) | (pp.PP_GRAD_ADD if add is not None else 0)
    pp.prunepath_route_topk_grad(dev(g), T, E, idx.shape[1], dev(idx, np.int32), dev(dw),
                                 c["scale"], flags, dg)
    torch.cuda.synchronize()
    dg = dg.cpu().numpy()
    assert (dg[T * E:] == -77).all()
    return dg[:T * E].reshape(T, E)


def grad_tolerance(g, idx, dw, c):
    """Of q (see weight_tolerance), of a - D and of sums over up to 256 slots (8 levels), all
    relative to the largest |a| of the row, which bounds every term."""
    a = np.where(idx >= 0, np.abs(np.nan_to_num(dw)), 0.0).max(1, keepdims=True)
    return (weight_tolerance(g, idx) * 3 + 16 * STEP) * a * abs(c["scale"]) + 1e-37


def check_grad(g, idx, dw, c):
    ref = op.route_topk_grad(g, idx, dw, c["scale"], c["sigmoid"], c["renorm"])
    tol = grad_tolerance(g, idx, dw, c)
    dg = grad(g, idx, dw, c)
    assert (np.abs(dg - ref) <= tol).all(), np.abs(dg - ref).max()
    add = logits(*g.shape, seed=77, std=0.5)
    both = grad(g, idx, dw, c, add)
    # the gradient's own rounding order may differ from the plain call's by fused additions
    assert (np.abs(both - (add.astype(np.float64) + ref)) <= tol + STEP * (np.abs(add) + np.abs(ref))).all()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 1), (3, 16, 16), (5, 17, 3), (65, 112, 8),
                                   (33, 148, 6), (2, 256, 256), (130, 256, 8), (4, 255, 33)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient(T, E, k, sigmoid, renorm):
    print("route_topk_grad T=%d E=%d k=%d" % (T, E, k), flush=True)
    g = logits(T, E, E + k)
    c = case(k, scale=1.5, sigmoid=sigmoid, renorm=renorm)
    idx, _ = route(g, c)
    check_grad(g, idx, logits(T, k, 3, 1.0), c)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_masked_rows_and_odd_choices(sigmoid, renorm):
    """Empty rows and slots (whose dgate_w is NaN), masked experts, saturated scores, indices out
    of range, an expert named twice."""
    rng = np.random.default_rng(14)
    g = logits(30, 40, 15)
    g[rng.random(g.shape) < 0.6] = -np.inf
    g[2] = -np.inf
    g[3] = np.nan
    g[4] = 90.0
    g[5] = -120.0
    g[6, 7] = np.inf
    c = case(12, scale=2.0, sigmoid=sigmoid, renorm=renorm)
    idx, _ = route(g, c)
    dw = logits(30, 12, 16, 1.0)
    dw[idx < 0] = np.nan
    check_grad(g, idx, dw, c)
    idx = idx.copy()
    idx[8, 0], idx[9, 1], idx[10, 2] = 40, 1 << 30, -(1 << 31)
    idx[11, :] = 5
    idx[12, :3] = idx[12, 0]
    check_grad(g, idx, np.nan_to_num(dw), c)


def test_gradient_against_differences_of_the_call():
    """Central differences of the forward call itself, in steps that keep the choice."""
    T, E, k = 6, 24, 4
    g = logits(T, E, 17, 1.0)
    for sigmoid in (False, True):
        for renorm in (False, True):
            c = case(k, sigmoid=sigmoid, renorm=renorm)
            idx, _ = route(g, c)
            dw = logits(T, k, 18, 1.0)
            dg = grad(g, idx, dw, c)
            h = np.float32(2.0 ** -8)
            for t in range(T):
                e = int(idx[t, 1])
                a, b = g.copy(), g.copy()
                a[t, e] += h
                b[t, e] -= h
                (ia, wa), (ib, wb) = route(a, c), route(b, c)
                if not (set(ia[t]) == set(ib[t]) == set(idx[t])):
                    continue
                d = {int(x): float(v) for x, v in zip(idx[t], dw[t])}
                fa = sum(d[int(x)] * float(v) for x, v in zip(ia[t], wa[t]))
                fb = sum(d[int(x)] * float(v) for x, v in zip(ib[t], wb[t]))
                # h^2 / 6 times a third derivative of at most 1 of each of 4 weights times |dw| < 4,
                # and fp32 errors of 1e-6 per weight over 2 h
                tol = 4 * 4 * (float(h) ** 2 / 6) + 4 * 4 * 1e-6 / (2 * float(h))
                assert abs((fa - fb) / (2 * float(h)) - dg[t, e]) <= tol


# ------------------------------------------------------------------ streams, graphs, handles

def test_replayed_graph_gives_the_eager_bits():
    import torch
    T, E, k = 777, 112, 8
    c = case(k, 4, 2, logits(1, E, 21, 0.1)[0], 1.0, True, True, True)
    g, bias, dw = dev(logits(T, E, 20)), dev(c["sel_bias"]), dev(logits(T, k, 22))
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    w, dg = torch.zeros((T, k), device="cuda"), torch.zeros((T, E), device="cuda")

    def both():
        pp.prunepath_route_topk_logits(g, T, E, k, 4, 2, bias, 1.0, flags_of(c), idx, w)
        pp.prunepath_route_topk_grad(g, T, E, k, idx, dw, 1.0, flags_of(c), dg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(3):
        g.copy_(dev(logits(T, E, 30 + seed)))
        both()
        eager = [a.clone() for a in (idx, w, dg)]
        for a in (idx, w, dg):
            a.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((idx, w, dg), eager):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls without a handle share nothing."""
    import torch
    T, E, k = 4000, 160, 6
    gs = [dev(logits(T, E, s)) for s in (1, 2)]
    c = case(k, sigmoid=True, renorm=True)
    want = [route(g.cpu().numpy(), c) for g in gs]
    streams = [torch.cuda.Stream() for _ in gs]
    outs = [(torch.zeros((T, k), dtype=torch.int32, device="cuda"),
             torch.zeros((T, k), device="cuda")) for _ in gs]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s, (i, w) in zip(gs, streams, outs):
            pp.prunepath_route_topk_logits(g, T, E, k, 1, 1, None, 1.0, flags_of(c), i, w, stream=s)
    torch.cuda.synchronize()
    for (i, w), (ri, rw) in zip(outs, want):
        np.testing.assert_array_equal(i.cpu().numpy(), ri)
        np.testing.assert_array_equal(w.cpu().numpy(), rw)


@pytest.mark.parametrize("T", [1, 5, 64, 65, 200])
def test_handle_route(T):
    """On a handle's router: the logits are W_r x (+ b) times inv_temp, the choice is that of the
    call on those logits bit for bit, and plain top-k is the layer's own PP_SELECT_TOPK choice."""
    import torch
    d, E, k = 576, 24, 5
    rng = np.random.default_rng(T)
    bf = lambda a: torch.from_numpy(a.astype(np.float32)).bfloat16().cuda()  # noqa: E731
    Wr, x = bf(rng.standard_normal((E, d)) * 3 / np.sqrt(d)), bf(rng.standard_normal((T, d)))
    Wg, Wu = bf(rng.standard_normal((128 * E, d)) * .02), bf(rng.standard_normal((128 * E, d)) * .02)
    Wd = bf(rng.standard_normal((d, 128 * E)) * .02)
    b, it = dev(rng.standard_normal(E)), dev(0.5 + rng.random(T))
    h = pp.prunepath_create(d, 128 * E, E, 256, Wr, Wg, Wu, Wd, router_bias=b,
                            flags=pp.PP_SELECT_TOPK)
    try:
        g = torch.full((T, E), float("nan"), device="cuda")
        idx, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
        pp.prunepath_route_topk(h, x, T, it, k, 1, 1, None, 1.0, pp.PP_TOPK_RENORM, idx, w, g)
        full = torch.zeros((T, E), dtype=torch.int32, device="cuda")
        cnt = torch.zeros((T,), dtype=torch.int32, device="cuda")
        pp.prunepath_route(h, x, T, float(k), it, full, cnt)
        i2, w2 = torch.zeros_like(idx), torch.zeros_like(w)
        pp.prunepath_route_topk(h, x, T, it, k, 1, 1, None, 1.0, pp.PP_TOPK_RENORM, i2, w2)
        torch.cuda.synchronize()
        assert torch.equal(full[:, :k], idx) and (cnt == k).all()
        assert torch.equal(i2, idx) and torch.equal(w2, w)
        ref = (x.double() @ Wr.double().t() + b.double()) * it.double()[:, None]
        # 576 exact products summed in fp32 in chains of 16 K-steps
        bound = 64 * 2.0 ** -24 * ((x.double().abs() @ Wr.double().abs().t()) + b.double().abs()) * it.double()[:, None]
        assert ((g.double() - ref).abs() <= bound).all()
        ri, rw = route(g.cpu().numpy(), case(k, renorm=True))
        np.testing.assert_array_equal(idx.cpu().numpy(), ri)
        np.testing.assert_array_equal(w.cpu().numpy(), rw)
    finally:
        pp.prunepath_destroy(h)


@pytest.mark.parametrize("T", [1, 3, 70])
@pytest.mark.parametrize("E,G,top", [(160, 1, 1), (160, 8, 3), (24, 1, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_handle_route_rules(T, E, G, top, sigmoid):
    """Biases, groups and many experts on a handle's router: the choice and the weights of the call
    on the logits that it reports, bit for bit (d 1088: three K-slices, the last of one K-step)."""
    import torch
    d, k = 1088, 6
    torch.manual_seed(T + E)
    bf = lambda *s: torch.randn(s, device="cuda").mul_(0.05).bfloat16()  # noqa: E731
    x = torch.randn((T, d), device="cuda").bfloat16()
    bias = torch.randn(E, device="cuda") * 0.1
    fl = (pp.PP_SCORE_SIGMOID if sigmoid else 0) | pp.PP_GROUP_TOP2
    h = pp.prunepath_create(d, 128 * E, E, 128, bf(E, d), bf(128 * E, d), bf(128 * E, d),
                            bf(d, 128 * E))
    try:
        for b in (None, bias):
            g = torch.full((T, E), float("nan"), device="cuda")
            idx, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
            i2, w2 = torch.ones_like(idx), torch.ones_like(w)
            pp.prunepath_route_topk(h, x, T, None, k, G, top, b, 1.5, fl, idx, w, g)
            pp.prunepath_route_topk_logits(g, T, E, k, G, top, b, 1.5, fl, i2, w2)
            assert torch.equal(idx, i2) and torch.equal(w, w2)
            ri, _ = op.route_topk(g.cpu().numpy(), k, G, top, None if b is None else b.cpu().numpy(),
                                  1.5, sigmoid, False, True)
            np.testing.assert_array_equal(idx.cpu().numpy(), ri)
    finally:
        torch.cuda.synchronize()
        pp.prunepath_destroy(h)


def test_handle_refusals():
    import torch
    d, E = 64, 2
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h = pp.prunepath_create(d, 128 * E, E, 4, z(E, d), z(128 * E, d), z(128 * E, d), z(d, 128 * E))
    try:
        i, w = torch.zeros((8, 2), dtype=torch.int32, device="cuda"), torch.zeros((8, 2), device="cuda")
        y = torch.zeros((8, d), device="cuda")
        lib = pp.load()
        p = [a.data_ptr() for a in (z(8, d), i, w, y)]
        for kw in (dict(T=0), dict(T=5), dict(k=0), dict(k=3), dict(x=None), dict(i=None)):
            a = dict(x=p[0], T=2, k=2, i=p[1])
            a.update(kw)
            assert lib.prunepath_route_topk(h, a["x"], a["T"], None, a["k"], 1, 1, None, 1.0, 0,
                                            a["i"], p[2], None, None) == pp.PP_EINVAL
            for f in (lib.prunepath_ffn_decode_routed, lib.prunepath_ffn_prefill_routed):
                assert f(h, a["x"], a["T"], a["k"], a["i"], p[2], p[3], None) == pp.PP_EINVAL
        for f in (lib.prunepath_ffn_decode_routed, lib.prunepath_ffn_prefill_routed):
            assert f(h, p[0], 2, 2, p[1], p[2], None, None) == pp.PP_EINVAL
            assert f(h, p[0], 2, 2, p[1] + 2, p[2], p[3], None) == pp.PP_EINVAL
    finally:
        pp.prunepath_destroy(h)


def test_binding_refuses_short_and_foreign_arrays():
    import torch
    g = torch.zeros((4, 8), device="cuda")
    i, w = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    with pytest.raises(ValueError):
        pp.prunepath_route_topk_logits(g, 5, 8, 2, 1, 1, None, 1.0, 0, i, w)
    with pytest.raises(ValueError):
        pp.prunepath_route_topk_logits(g, 4, 8, 4, 1, 1, None, 1.0, 0, i, w)
    with pytest.raises(ValueError):
        pp.prunepath_route_topk_logits(g.cpu(), 4, 8, 2, 1, 1, None, 1.0, 0, i, w)
    with pytest.raises(ValueError):
        pp.prunepath_route_topk_logits(g.t(), 8, 4, 1, 1, 1, None, 1.0, 0, i, w)
    with pytest.raises(TypeError):
        pp.prunepath_route_topk_logits(g, 4, 8, 2, 1, 1, None, 1.0, 0, i.float(), w)
