"""Arrays of the routing calls that are the same: refused before any HIP call (runs without a GPU
but for the call on a handle)."""
import pytest

import paper_2605_28283_amd as pp


@pytest.mark.parametrize("g,bias,idx,w", [(16, 32, 16, 64), (16, 32, 48, 16), (16, 32, 32, 64),
                                          (16, 32, 48, 32), (16, None, 48, 48)])
def test_route_topk_logits_refuses_shared_arrays(g, bias, idx, w):
    assert pp.load().prunepath_route_topk_logits(g, 8, 64, 4, 8, 4, bias, 1.0, 0, idx, w,
                                                 None) == pp.PP_EINVAL


@pytest.mark.gpu
def test_handle_call_refuses_shared_arrays():
    import torch
    d, E = 64, 2
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h = pp.prunepath_create(d, 128 * E, E, 4, z(E, d), z(128 * E, d), z(128 * E, d), z(d, 128 * E))
    try:
        own = [torch.zeros(256, device="cuda") for _ in range(5)]
        x, bias, idx, w, g = (a.data_ptr() for a in own)
        f = lambda x, bias, idx, w, g: pp.load().prunepath_route_topk(  # noqa: E731
            h, x, 4, None, 2, 1, 1, bias, 1.0, 0, idx, w, g, None)
        for bad in ((x, bias, x, w, g), (x, bias, idx, x, g), (x, bias, idx, w, x),
                    (x, bias, bias, w, g), (x, bias, idx, bias, g), (x, bias, idx, w, bias),
                    (x, bias, idx, w, idx), (x, bias, idx, w, w)):
            assert f(*bad) == pp.PP_EINVAL
        assert f(x, bias, idx, w, g) == pp.PP_OK
        assert f(x, None, idx, w, None) == pp.PP_OK
        torch.cuda.synchronize()
    finally:
        pp.prunepath_destroy(h)


@pytest.mark.gpu
def test_handle_call_refuses_outputs_in_the_temperatures():
    import torch
    d, E = 64, 2
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h = pp.prunepath_create(d, 128 * E, E, 4, z(E, d), z(128 * E, d), z(128 * E, d), z(d, 128 * E))
    try:
        own = [torch.ones(256, device="cuda") for _ in range(5)]
        x, it, idx, w, g = (a.data_ptr() for a in own)
        f = lambda idx, w, g: pp.load().prunepath_route_topk(  # noqa: E731
            h, x, 4, it, 2, 1, 1, None, 1.0, 0, idx, w, g, None)
        assert f(it, w, g) == f(idx, it, g) == f(idx, w, it) == pp.PP_EINVAL
        assert f(idx, w, g) == f(idx, w, None) == pp.PP_OK
        torch.cuda.synchronize()
    finally:
        pp.prunepath_destroy(h)


@pytest.mark.gpu
def test_handle_call_refuses_misaligned_arrays():
    """fp32 and int32 arrays lie on 4 bytes, the temperatures among them."""
    import torch
    d, E = 64, 2
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    h = pp.prunepath_create(d, 128 * E, E, 4, z(E, d), z(128 * E, d), z(128 * E, d), z(d, 128 * E))
    try:
        own = [torch.ones(256, device="cuda") for _ in range(6)]
        at = [a.data_ptr() for a in own]
        for bad in (None, 1, 2, 3, 4, 5):
            x, it, bias, idx, w, g = (p + (2 if i == bad else 0) for i, p in enumerate(at))
            st = pp.load().prunepath_route_topk(h, x, 4, it, 2, 1, 1, bias, 1.0, 0, idx, w, g, None)
            assert st == (pp.PP_OK if bad is None else pp.PP_EINVAL)
        torch.cuda.synchronize()
    finally:
        pp.prunepath_destroy(h)
