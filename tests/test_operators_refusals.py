"""Argument checks of the routing to a fixed number of experts, the routed experts' products and
the residual layer norm: every call here returns before any HIP call (runs without a GPU).  The
fp64 forms that the GPU tests compare with are pinned here too, by brute force and differences."""
import numpy as np
import pytest
import torch

import paper_2605_28283_amd as pp
from oracle import operators as op
from paper_2605_28283_amd.stack import DecodeStack

INF, NAN = float("inf"), float("nan")
MANY = pp.PP_SCORE_SIGMOID | pp.PP_TOPK_RENORM | pp.PP_GROUP_TOP2


def logits_call(g=16, T=8, E=64, k=4, G=8, top=4, bias=32, scale=1.0, flags=MANY, idx=48, w=64):
    return pp.load().prunepath_route_topk_logits(g, T, E, k, G, top, bias, scale, flags, idx, w,
                                                 None)


BAD_RULE = [dict(k=0), dict(k=33), dict(k=-1), dict(G=0), dict(G=3), dict(G=-8), dict(top=0),
            dict(top=9), dict(bias=33), dict(scale=NAN), dict(scale=INF), dict(scale=-INF),
            dict(flags=16), dict(flags=pp.PP_GRAD_ADD), dict(idx=None), dict(w=None), dict(idx=50),
            dict(w=65), dict(w=48)]


@pytest.mark.parametrize("kw", BAD_RULE + [
    dict(g=None), dict(g=18), dict(T=0), dict(T=(1 << 22) + 1), dict(E=0), dict(E=257, G=1, top=1),
    dict(T=-1), dict(E=-8)])
def test_route_topk_logits_refuses(kw):
    assert logits_call(**kw) == pp.PP_EINVAL


def test_route_topk_refuses_many_groups():
    assert logits_call(E=64, G=32, top=32) == pp.PP_EUNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(g=None), dict(idx=None), dict(dw=None), dict(dg=None), dict(dg=16), dict(dg=64),
    dict(dg=48), dict(g=17), dict(idx=49), dict(dw=66), dict(dg=81), dict(T=0),
    dict(T=(1 << 22) + 1), dict(E=0), dict(E=257), dict(k=0), dict(k=65), dict(scale=NAN),
    dict(flags=16)])
def test_route_topk_grad_refuses(kw):
    a = dict(g=16, T=8, E=64, k=4, idx=48, dw=64, scale=1.0, flags=0, dg=80)
    a.update(kw)
    assert pp.load().prunepath_route_topk_grad(a["g"], a["T"], a["E"], a["k"], a["idx"], a["dw"],
                                               a["scale"], a["flags"], a["dg"],
                                               None) == pp.PP_EINVAL


def test_handle_calls_refuse_null_handle():
    lib = pp.load()
    assert lib.prunepath_route_topk(None, 16, 1, None, 1, 1, 1, None, 1.0, 0, 16, 32, None,
                                    None) == pp.PP_EINVAL
    for f in (lib.prunepath_ffn_decode_routed, lib.prunepath_ffn_prefill_routed):
        assert f(None, 16, 1, 1, 16, 32, 48, None) == pp.PP_EINVAL


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(u=None), dict(T=0), dict(T=(1 << 20) + 1), dict(d=0), dict(d=65537),
    dict(eps=NAN), dict(eps=-1e-5), dict(eps=INF), dict(flags=2), dict(x=18), dict(y=33),
    dict(x_out=50), dict(w=65), dict(b=81), dict(u=97), dict(stats=114), dict(u=16), dict(u=32),
    dict(u=48), dict(u=98, flags=pp.PP_NORM_F32)])
def test_layernorm_refuses(kw):
    a = dict(x=16, y=32, x_out=48, T=4, d=8, eps=1e-5, w=64, b=80, u=96, stats=112, flags=0)
    a.update(kw)
    assert pp.load().prunepath_residual_layernorm(
        a["x"], a["y"], a["x_out"], a["T"], a["d"], a["eps"], a["w"], a["b"], a["u"], a["stats"],
        a["flags"], None) == pp.PP_EINVAL


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(du=None), dict(stats=None), dict(dx=None), dict(ws=None),
    dict(ws=None, db=None), dict(T=0), dict(T=(1 << 20) + 1), dict(d=0), dict(d=65537),
    dict(flags=2), dict(x=18), dict(du=33), dict(du=34, flags=pp.PP_NORM_F32), dict(dres=49),
    dict(w=65), dict(stats=81), dict(dx=98), dict(dw=114), dict(db=129), dict(ws=146), dict(dx=16),
    dict(dx=32), dict(db=112)])
def test_layernorm_grad_refuses(kw):
    a = dict(x=16, du=32, dres=48, T=4, d=8, w=64, stats=80, dx=96, dw=112, db=128, ws=144,
             flags=0)
    a.update(kw)
    assert pp.load().prunepath_residual_layernorm_grad(
        a["x"], a["du"], a["dres"], a["T"], a["d"], a["w"], a["stats"], a["dx"], a["dw"], a["db"],
        a["ws"], a["flags"], None) == pp.PP_EINVAL


def test_layernorm_grad_workspace():
    size = pp.prunepath_residual_layernorm_grad_workspace
    for T, d in ((1, 1), (1, 65536), (1 << 20, 1), (1 << 20, 65536), (33, 4096)):
        assert size(T, d) > 0 and size(T, d) % 4 == 0
    for T, d in ((0, 8), (8, 0), (-1, 8), ((1 << 20) + 1, 8), (8, 65537)):
        assert size(T, d) == 0


def test_stack_refuses():
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, norms=[(None, None)])
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, topk=dict(k=1, groups=2))
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, topk=dict(n_groups=2))
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, topk=dict(k=1, sel_bias=[None]))


def test_stack_refuses_short_selection_bias():
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, topk=dict(k=1, sel_bias=[None, torch.zeros(3)]))
    with pytest.raises(ValueError):
        DecodeStack([1], 64, 2, 1, 0.5, topk=dict(k=1, sel_bias=[torch.zeros(1)]))


# ------------------------------------------------------------------ the fp64 forms

@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_reference_gradient_is_the_difference_quotient(sigmoid, renorm):
    rng = np.random.default_rng(3)
    g = rng.standard_normal((3, 12)) * 2
    g[1, 4] = -np.inf
    idx, _ = op.route_topk(g, 4, sigmoid=sigmoid, renorm=renorm)
    dw = rng.standard_normal(idx.shape)
    dg = op.route_topk_grad(g, idx, dw, 2.5, sigmoid, renorm)

    def loss(z):
        total = 0.0
        for t in range(len(z)):
            s = np.exp(op.log_scores(z[t], sigmoid))[idx[t]]
            total += 2.5 * ((s / s.sum() if renorm else s) * dw[t]).sum()
        return total
    h = 1e-6
    for t in range(3):
        for e in range(12):
            if np.isinf(g[t, e]):
                assert dg[t, e] == 0.0
                continue
            a, b = g.copy(), g.copy()
            a[t, e] += h
            b[t, e] -= h
            # central difference: h^2 / 6 of a third derivative of order 10, 1e-16 / h rounding
            assert abs((loss(a) - loss(b)) / (2 * h) - dg[t, e]) <= 1e-8


def test_reference_norm_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(4)
    r, du, dres = (rng.standard_normal((2, 7)) for _ in range(3))
    w = 1 + 0.3 * rng.standard_normal(7)
    dx, dw, db = op.layernorm_grad(r, du, dres, 1e-5, w)
    f = lambda r, w, b: (op.layernorm(r, 1e-5, w, b)[0] * du).sum() + (r * dres).sum()  # noqa: E731
    h = 1e-6
    for i in np.ndindex(2, 7):
        a, b = r.copy(), r.copy()
        a[i] += h
        b[i] -= h
        assert abs((f(a, w, 0 * w) - f(b, w, 0 * w)) / (2 * h) - dx[i]) <= 1e-7
    for j in range(7):
        e = np.eye(7)[j] * h
        assert abs((f(r, w + e, 0 * w) - f(r, w - e, 0 * w)) / (2 * h) - dw[j]) <= 1e-7
        assert abs((f(r, w, e) - f(r, w, -e)) / (2 * h) - db[j]) <= 1e-7


def test_reference_choice_by_brute_force():
    """Among all choices of groups and of experts in them, the reference's has the largest sums."""
    import itertools
    rng = np.random.default_rng(5)
    for _ in range(20):
        g, bias = rng.standard_normal((1, 12)) * 2, rng.standard_normal(12) * 0.2
        idx, _ = op.route_topk(g, 3, 4, 2, bias, sigmoid=True, top2=True)
        c = 1 / (1 + np.exp(-g[0])) + bias
        worth = [np.sort(c[3 * a:3 * a + 3])[-2:].sum() for a in range(4)]
        groups = max(itertools.combinations(range(4), 2), key=lambda s: sum(worth[a] for a in s))
        allowed = [e for e in range(12) if e // 3 in groups]
        best = max(itertools.combinations(allowed, 3), key=lambda s: sum(c[e] for e in s))
        assert sorted(idx[0]) == sorted(best)
        assert (np.diff(c[idx[0]]) <= 0).all()
