"""The experts' products on a given choice, against the plain fp64 form (whose bound on the kernels'
roundings oracle.operators.routed_ffn derives) and against the layer's own routed calls; and the
routing, the products and the layer norm run together, as a stack's layer does."""
import numpy as np
import pytest

import paper_2605_28283_amd as pp
from oracle import operators as op

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, d, E, max_tokens, mlp=False, flags=0, seed=0, biases=True):
        import torch
        rng = np.random.default_rng(seed)
        r = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
        bf = lambda a: torch.from_numpy(a).bfloat16().cuda()  # noqa: E731
        self.d, self.E, self.mlp = d, E, mlp
        self.Wr = bf(r(E, d) * 3 / np.sqrt(d).astype(np.float32))
        self.Win, self.Wout = bf(r(128 * E, d) * .05), bf(r(d, 128 * E) * .05)
        self.Wup, self.b_in, self.b_out = None, None, None
        if mlp:
            if biases:
                self.b_in = torch.from_numpy(r(128 * E) * np.float32(.1)).cuda()
                self.b_out = torch.from_numpy(r(d) * np.float32(.1)).cuda()
            self.h = pp.prunepath_create_mlp(d, 128 * E, E, max_tokens, self.Wr, self.Win,
                                             self.b_in, self.Wout, self.b_out, flags=flags)
        else:
            self.Wup = bf(r(128 * E, d) * .05)
            self.h = pp.prunepath_create(d, 128 * E, E, max_tokens, self.Wr, self.Win, self.Wup,
                                         self.Wout, flags=flags)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        import torch
        torch.cuda.synchronize()
        pp.prunepath_destroy(self.h)

    def reference(self, x, idx, w):
        f = lambda a: None if a is None else a.float().cpu().numpy()  # noqa: E731
        return op.routed_ffn(f(x), idx, w, f(self.Win), f(self.Wup), f(self.Wout), f(self.b_in),
                             f(self.b_out))

    def run(self, x, idx, w, prefill, guard=5):
        import torch
        T, k = idx.shape
        y = torch.full((T * self.d + guard,), -77.0, device="cuda")
        f = pp.prunepath_ffn_prefill_routed if prefill else pp.prunepath_ffn_decode_routed
        f(self.h, x, T, k, torch.from_numpy(np.ascontiguousarray(idx, np.int32)).cuda(),
          None if w is None else torch.from_numpy(np.ascontiguousarray(w, np.float32)).cuda(), y)
        torch.cuda.synchronize()
        y = y.cpu().numpy()
        assert (y[T * self.d:] == -77).all()
        return y[:T * self.d].reshape(T, self.d)


def tokens(T, d, seed=1):
    import torch
    x = np.random.default_rng(seed).standard_normal((T, d)).astype(np.float32)
    return torch.from_numpy(x).bfloat16().cuda()


def choices(T, E, k, seed=2, holes=0.0):
    rng = np.random.default_rng(seed)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    w = rng.standard_normal((T, k)).astype(np.float32)
    hole = rng.random((T, k)) < holes
    idx[hole] = -1
    w[hole] = np.nan
    return idx, w


def check(L, x, idx, w, prefill):
    print("routed T=%d k=%d d=%d E=%d prefill=%d" % (*idx.shape, L.d, L.E, prefill), flush=True)
    y = L.run(x, idx, w, prefill)
    ref, bound = L.reference(x, idx, w)
    assert (np.abs(y - ref) <= bound + 2.0 ** -23 * np.abs(ref)).all(), \
        np.nanmax(np.abs(y - ref) / (bound + 1e-30))
    return y


@pytest.mark.parametrize("mlp", [False, True])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 4), (1, 24), (3, 2), (17, 5), (64, 3), (65, 4),
                                 (200, 2), (64, 24)])
def test_products(mlp, T, k):
    with Layer(320, 24, 256, mlp) as L:
        x = tokens(T, 320, T)
        idx, w = choices(T, 24, k, T + k, holes=0.1)
        a = check(L, x, idx, w, False)
        b = check(L, x, idx, w, True)
        check(L, x, idx, None, T % 2 == 0)
        # again, with other work of the handle in between: the same bits
        check(L, tokens(5, 320, 9), *choices(5, 24, 3, 1), prefill=False)
        assert L.run(x, idx, w, False).tobytes() == a.tobytes()
        assert L.run(x, idx, w, True).tobytes() == b.tobytes()


@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("mlp", [False, True])
def test_odd_choices(mlp, prefill):
    """Nobody's expert, tokens without one, indices out of range, an expert twice, weights 0 and
    negative, every token on one expert."""
    with Layer(128, 12, 128, mlp, flags=pp.PP_AGG_SIGMOID | pp.PP_SELECT_STRICT) as L:
        for T in (1, 2, 70, 128):
            x = tokens(T, 128, T)
            idx = np.full((T, 4), -1, np.int32)
            w = np.full((T, 4), np.nan, np.float32)
            y = check(L, x, idx, w, prefill)
            assert (y == (0 if L.b_out is None else L.b_out.cpu().numpy())).all()
            idx[T // 2] = [12, 1 << 30, -(1 << 31), 255]
            check(L, x, idx, w, prefill)
            idx[:] = 7
            w[:] = [0.5, -1.25, 3.0, 0.125]
            check(L, x, idx, w, prefill)
            idx[:, 1] = 3
            w[0] = 0.0
            check(L, x, idx, w, prefill)
            idx[:] = [2, 11, 2, 0]
            check(L, x, idx, w, prefill)
            check(L, x, idx, None, prefill)


@pytest.mark.parametrize("flags", [0, pp.PP_AGG_SIGMOID])
@pytest.mark.parametrize("mlp", [False, True])
@pytest.mark.parametrize("T", [1, 2, 33, 64, 200])
def test_the_layers_own_choice_gives_the_layers_own_bits(flags, mlp, T):
    """idx and weights as prunepath_route reports them, through the routed calls: y is that of
    prunepath_ffn_decode and _prefill, whose kernels these are."""
    import torch
    d, E, tau = 256, 20, 0.8
    with Layer(d, E, 256, mlp, flags) as L:
        x = tokens(T, d, T)
        full = torch.zeros((T, E), dtype=torch.int32, device="cuda")
        cnt, gw = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros((T, E), device="cuda")
        pp.prunepath_route(L.h, x, T, tau, None, full, cnt, gw)
        for own, routed in ((pp.prunepath_ffn_decode, pp.prunepath_ffn_decode_routed),
                            (pp.prunepath_ffn_prefill, pp.prunepath_ffn_prefill_routed)):
            a, b = torch.zeros((T, d), device="cuda"), torch.ones((T, d), device="cuda")
            own(L.h, x, T, tau, None, a)
            routed(L.h, x, T, E, full, gw, b)
            assert torch.equal(a, b)


def test_own_calls_after_routed_ones_are_unchanged():
    import torch
    d, E, T = 192, 16, 40
    with Layer(d, E, 64) as L:
        x, y1, y2 = tokens(T, d), torch.zeros((T, d), device="cuda"), torch.zeros((T, d), device="cuda")
        for f in (pp.prunepath_ffn_decode, pp.prunepath_ffn_prefill):
            f(L.h, x, T, 0.7, None, y1)
            L.run(x, *choices(T, E, E), prefill=False)
            L.run(x, *choices(T, E, 1), prefill=True)
            f(L.h, x, T, 0.7, None, y2)
            torch.cuda.synchronize()
            assert torch.equal(y1, y2)


@pytest.mark.parametrize("prefill", [False, True])
def test_a_wide_layer(prefill):
    """A benchmark-shaped layer (4096 wide, 112 experts), some rows compared."""
    d, E, T, k = 4096, 112, 48, 8
    with Layer(d, E, T, seed=3) as L:
        x = tokens(T, d, 5)
        x = x * 0.25
        idx, w = choices(T, E, k, 6)
        y = L.run(x, idx, w, prefill)
        rows = [0, 17, 47]
        ref, bound = L.reference(x[rows], idx[rows], w[rows])
        assert (np.abs(y[rows] - ref) <= bound + 2.0 ** -23 * np.abs(ref)).all()


@pytest.mark.parametrize("T,prefill", [(1, False), (48, False), (150, True)])
@pytest.mark.parametrize("mlp", [False, True])
def test_a_layer_as_it_is_served(T, prefill, mlp):
    """Norm, router, choice, products, residual add and the next norm: eager, and captured in a
    graph that is replayed on new tokens with eager work in between; each step checked on the
    inputs that it had."""
    import torch
    d, E, k, G, top = 256, 24, 4, 4, 2
    flags = pp.PP_SCORE_SIGMOID | pp.PP_TOPK_RENORM | pp.PP_GROUP_TOP2
    rng = np.random.default_rng(7)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    with Layer(d, E, T, mlp) as L:
        x, w, b, bias = f(T, d) * 4, 1 + f(d) * .1, f(d) * .1, f(E) * .05
        u0, u1 = (torch.zeros((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        idx, gw, g = torch.zeros((T, k), dtype=torch.int32, device="cuda"), z(T, k), z(T, E)
        y, x1 = z(T, d), z(T, d)
        ffn = pp.prunepath_ffn_prefill_routed if prefill else pp.prunepath_ffn_decode_routed

        def layer():
            pp.prunepath_residual_layernorm(x, None, None, T, d, 1e-5, w, b, u0)
            pp.prunepath_route_topk(L.h, u0, T, None, k, G, top, bias, 2.5, flags, idx, gw, g)
            ffn(L.h, u0, T, k, idx, gw, y)
            pp.prunepath_residual_layernorm(x, y, x1, T, d, 1e-5, w, b, u1)
        layer()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer()
        outs = (u0, idx, gw, g, y, x1, u1)
        for rep in range(3):
            x.copy_(f(T, d) * 4)
            layer()
            eager = [a.clone() for a in outs]
            for a in outs:
                a.fill_(3)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, e in zip(outs, eager):
                assert torch.equal(a, e)
        n = lambda a: a.float().cpu().numpy()  # noqa: E731
        ru, _, _ = op.layernorm(n(x), 1e-5, n(w), n(b))
        assert (np.abs(n(u0) - ru) <= 2.0 ** -8 * np.abs(ru) + 1e-5).all()
        ri, rw = op.route_topk(n(g), k, G, top, n(bias), 2.5, True, True, True)
        np.testing.assert_array_equal(idx.cpu().numpy(), ri)
        assert (np.abs(n(gw) - rw) <= 1e-5 * rw).all()
        ref, bound = L.reference(u0, ri, n(gw))
        assert (np.abs(n(y) - ref) <= bound + 2.0 ** -23 * np.abs(ref)).all()
        np.testing.assert_array_equal(n(x1), n(x) + n(y))


def test_a_routers_training_step():
    """Norm, choice, regularisers, gradients of the weights' loss onto theirs, back through the
    router's product (a caller's own) and the norm: every gradient against differences of the
    whole chain in 64 bits."""
    import torch
    T, d, E, k = 24, 96, 16, 3
    rng = np.random.default_rng(9)
    r = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    x, w, b, Wr, dw = r(T, d), 1 + r(d) * np.float32(.1), r(d) * np.float32(.1), r(E, d) * np.float32(.2), r(T, k)
    eps, eta, lam, gam = 1e-8, 0.3, 0.2, 0.1
    D = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    xd, wd, u, st = D(x), D(w), z(T, d), z(T, 2)
    pp.prunepath_residual_layernorm(xd, None, None, T, d, 1e-5, wd, D(b), u, st, pp.PP_NORM_F32)
    g = (u.double() @ D(Wr).double().t()).float().contiguous()
    idx, gw, dg, losses = torch.zeros((T, k), dtype=torch.int32, device="cuda"), z(T, k), z(T, E), z(4)
    ws = torch.zeros(pp.prunepath_router_loss_workspace(T, E), dtype=torch.uint8, device="cuda")
    flags = pp.PP_SCORE_SOFTMAX | pp.PP_TOPK_RENORM
    pp.prunepath_router_loss(g, T, E, eps, eta, lam, gam, losses, dg, ws)
    pp.prunepath_route_topk_logits(g, T, E, k, 1, 1, None, 1.0, flags, idx, gw)
    pp.prunepath_route_topk_grad(g, T, E, k, idx, D(dw), 1.0, flags | pp.PP_GRAD_ADD, dg)
    du = (dg.double() @ D(Wr).double()).float().contiguous()
    dx, dwn, dbn = z(T, d), z(d), z(d)
    ws = torch.zeros(pp.prunepath_residual_layernorm_grad_workspace(T, d), dtype=torch.uint8,
                     device="cuda")
    pp.prunepath_residual_layernorm_grad(xd, du, None, T, d, wd, st, dx, dwn, dbn, ws,
                                         pp.PP_NORM_F32)
    torch.cuda.synchronize()
    ri = idx.cpu().numpy()

    def loss(x, w, b):
        u = op.layernorm(x, 1e-5, w, b)[0]
        z = u @ Wr.astype(np.float64).T
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        q = np.take_along_axis(p, ri.astype(np.int64), 1)
        q = q / q.sum(1, keepdims=True)
        reg = (-eta * (p * np.log(p + eps)).sum(1).mean() + lam * E * (p.mean(0) ** 2).sum() +
               gam * (1 / (1 + np.exp(-z))).mean())
        return reg + (q * dw).sum()
    h = 1e-5
    x, w, b = (a.astype(np.float64) for a in (x, w, b))
    # differences: h^2 times third derivatives of order 10, and 1e-14 / h; the kernels: some tens of
    # fp32 roundings of terms of order 1
    tol = 2e-5
    for t, j in ((0, 0), (5, 17), (23, 95)):
        e = np.zeros_like(x)
        e[t, j] = h
        assert abs((loss(x + e, w, b) - loss(x - e, w, b)) / (2 * h) - float(dx[t, j])) <= tol
    for j in (0, 50):
        e = np.eye(d)[j] * h
        assert abs((loss(x, w + e, b) - loss(x, w - e, b)) / (2 * h) - float(dwn[j])) <= 5 * tol
        assert abs((loss(x, w, b + e) - loss(x, w, b - e)) / (2 * h) - float(dbn[j])) <= 5 * tol
