"""The binding's calls on a handle know the layer's sizes: an array that is shorter than what the
call touches is refused before the library is asked (a stand-in for it here, and for the tensors:
runs without a GPU)."""
import pytest
import torch

import paper_2605_28283_amd as pp
from paper_2605_28283_amd import _lib

D, E, T, K = 64, 6, 5, 3
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Array:
    """What the binding asks of a GPU tensor."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, n, dtype):
        self.n, self.dtype = n, dtype

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def numel(self):
        return self.n

    def data_ptr(self):
        return 4096


class Library:
    """Records the calls that reach it; every one succeeds."""

    def __init__(self):
        self.calls, self.made = [], 0

    def __getattr__(self, name):
        def call(*a):
            self.calls.append(name)
            if name in ("prunepath_create", "prunepath_create_mlp"):
                self.made += 1
                a[0]._obj.value = 1000 + self.made
            return pp.PP_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(_lib, "_current", (lambda: 0, lambda i: 0))
    monkeypatch.setattr(_lib, "_dims", {}, raising=False)
    return lib


def make(mlp):
    if mlp:
        return pp.prunepath_create_mlp(D, 128 * E, E, 8, 1, 1, None, 1, None)
    return pp.prunepath_create(D, 128 * E, E, 8, 1, 1, 1, 1)


SIZES = dict(x=T * D, inv_temp=T, sel_bias=E, idx=T * K, w=T * K, logits=T * E, y=T * D)
TYPES = dict(x=BF, idx=I32)


def call(name, h, **short):
    a = {n: Array(short.get(n, size), TYPES.get(n, F32)) for n, size in SIZES.items()}
    if name == "route":
        pp.prunepath_route_topk(h, a["x"], T, a["inv_temp"], K, 1, 1, a["sel_bias"], 1.0, 0,
                                a["idx"], a["w"], a["logits"])
    else:
        f = pp.prunepath_ffn_decode_routed if name == "decode" else pp.prunepath_ffn_prefill_routed
        f(h, a["x"], T, K, a["idx"], a["w"], a["y"])


CALLS = [("route", n) for n in ("x", "inv_temp", "sel_bias", "idx", "w", "logits")] + \
    [(f, n) for f in ("decode", "prefill") for n in ("x", "idx", "w", "y")]


@pytest.mark.parametrize("mlp", [False, True])
@pytest.mark.parametrize("name,short", CALLS)
def test_short_arrays_are_refused(lib, mlp, name, short):
    h = make(mlp)
    del lib.calls[:]
    with pytest.raises(ValueError):
        call(name, h, **{short: SIZES[short] - 1})
    assert lib.calls == []
    call(name, h)
    assert len(lib.calls) == 1


def test_sizes_are_those_of_the_handle(lib):
    """Each of two handles has its own, an address that is used again those of its new layer, and
    a handle made elsewhere asks nothing."""
    a, b = make(False), pp.prunepath_create(2 * D, 128, 1, 8, 1, 1, 1, 1)
    call("route", a)
    with pytest.raises(ValueError):
        call("route", b)
    pp.prunepath_destroy(a)
    lib.made = 0
    assert pp.prunepath_create(D // 2, 128 * E, E, 8, 1, 1, 1, 1) == a
    call("route", a, x=T * D // 2)
    call("route", 77, x=1)
