"""DecodeStack with layer norms and a fixed number of experts: each layer's steps on the inputs that
they had (the norm in fp64, the choice by the call on the layer's input, the products in fp64 with
the rounding bound of oracle.operators.routed_ffn), and graph replays against the eager step."""
import numpy as np
import pytest

import paper_2605_28283_amd as pp
from oracle import operators as op
from paper_2605_28283_amd.stack import DecodeStack
from test_gpu_routed import Layer

pytestmark = pytest.mark.gpu

D, E, K = 192, 16, 3
FLAGS = pp.PP_SCORE_SIGMOID | pp.PP_TOPK_RENORM | pp.PP_GROUP_TOP2


def n(a):
    return a.float().cpu().numpy()


@pytest.mark.parametrize("T", [1, 7, 64])
@pytest.mark.parametrize("mlp", [False, True])
@pytest.mark.parametrize("normed,routed", [(True, True), (True, False), (False, True)])
def test_stack(T, mlp, normed, routed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    layers = [Layer(D, E, 64, mlp, seed=l) for l in range(3)]
    try:
        norms = [(1 + 0.1 * f(D), None if l == 1 else 0.1 * f(D)) for l in range(3)]
        bias = [None if l == 1 else 0.05 * f(E) for l in range(3)]
        topk = dict(k=K, n_groups=4, top_groups=2, scale=1.5, flags=FLAGS, sel_bias=bias)
        st = DecodeStack([L.h for L in layers], D, E, T, 0.8, norms=norms if normed else None,
                         topk=topk if routed else None)
        st.set_input(4 * f(T, D))
        st.enqueue()
        torch.cuda.synchronize()
        for l, L in enumerate(layers):
            x, u, y = n(st.xs[l]), st.us[l].view(torch.bfloat16), n(st.ys[l])
            w, b = norms[l]
            r = x.astype(np.float64)
            ref = (op.layernorm(r, 1e-5, n(w), None if b is None else n(b))[0] if normed else
                   r / np.sqrt((r ** 2).mean(1, keepdims=True) + 1e-5))
            # half a bf16 step, and some tens of fp32 roundings of values up to about 5
            assert (np.abs(n(u) - ref) <= 2.0 ** -8 * np.abs(ref) + 2e-5).all()
            if routed:
                idx, gw = torch.zeros_like(st.idx[l]), torch.zeros_like(st.gate_w[l])
                pp.prunepath_route_topk(L.h, st.us[l], T, None, K, 4, 2, bias[l], 1.5, FLAGS, idx,
                                        gw)
                assert torch.equal(idx, st.idx[l]) and torch.equal(gw, st.gate_w[l])
                want, bound = L.reference(u, idx.cpu().numpy(), n(gw))
            else:
                want, bound = L.reference(u, st.idx[l].cpu().numpy(), None)
            assert (np.abs(y - want) <= bound + 2.0 ** -23 * np.abs(want)).all()
            np.testing.assert_array_equal(n(st.xs[l + 1]), x + y)
        eager = st.output.clone()
        st.capture()
        for rep in range(3):
            st.xs[1:].fill_(-1)
            st.replay()
            torch.cuda.synchronize()
            assert torch.equal(st.output, eager)
        x = 4 * f(T, D)
        st.set_input(x)
        st.replay()
        replayed = st.output.clone()
        st.enqueue()
        assert torch.equal(st.output, replayed) and not torch.equal(replayed, eager)
    finally:
        torch.cuda.synchronize()
        st.graph = None
        for L in layers:
            pp.prunepath_destroy(L.h)
