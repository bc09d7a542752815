"""The routing gradient at every number of columns that a lane can have, and one expert to either
side of it."""
import pytest

from test_gpu_topk import case, check_grad, logits, route

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("columns", range(1, 17))
@pytest.mark.parametrize("sigmoid,renorm", [(False, False), (True, False), (True, True)])
def test_gradient_widths(columns, sigmoid, renorm):
    for E in {16 * columns - 15, 16 * columns - 1, 16 * columns}:
        k = min(E, 6)
        print("E=%d k=%d" % (E, k), flush=True)
        g, c = logits(19, E, E), case(k, scale=1.5, sigmoid=sigmoid, renorm=renorm)
        idx, _ = route(g, c)
        check_grad(g, idx, logits(19, k, 3, 1.0), c)
