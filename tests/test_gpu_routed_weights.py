"""The experts' products with weights that are no numbers: the token that has one gets no numbers,
whatever the NaN's bits, and the others keep theirs."""
import numpy as np
import pytest

from test_gpu_routed import Layer, choices, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("mlp", [False, True])
@pytest.mark.parametrize("T", [1, 9, 70])
def test_nan_and_infinite_weights(T, mlp, prefill):
    print("T=%d mlp=%d prefill=%d" % (T, mlp, prefill), flush=True)
    with Layer(128, 12, 128, mlp) as L:
        x = tokens(T, 128, T)
        idx, w = choices(T, 12, 3, T)
        plain = L.run(x, idx, w, prefill)
        t = T // 2
        for bits in (0x7FC00000, 0x7FFFFFFF, 0xFFFFFFFF, 0xFFC00000, 0x7F800001, 0x7F800000,
                     0xFF800000):
            v = w.copy()
            v.view(np.uint32)[t, 1] = bits
            y = L.run(x, idx, v, prefill)
            assert np.isnan(y[t]).all(), hex(bits)
            assert np.delete(y, t, 0).tobytes() == np.delete(plain, t, 0).tobytes()
            again = idx.copy()
            again[t, 2] = again[t, 1]                       # the weight is one of a sum
            assert np.isnan(L.run(x, again, v, prefill)[t]).all(), hex(bits)
