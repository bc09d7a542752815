"""What DecodeStack takes as norms and selection biases."""
import pytest
import torch

from paper_2605_28283_amd.stack import DecodeStack


@pytest.mark.parametrize("norms", [
    [None, None], [(None, None), None], [(torch.ones(64), None), torch.ones(64)],
    [(torch.ones(64), None), (torch.ones(64),)], [(None, None), (None, torch.ones(65))],
    [(torch.ones(63), None), (None, None)]])
def test_norms_that_are_no_pairs_of_the_width(norms):
    """Refused as the stack is made, not by a step."""
    with pytest.raises(ValueError):
        DecodeStack([1, 2], 64, 2, 1, 0.5, norms=norms)


@pytest.mark.gpu
def test_no_biases_and_no_norm_weights():
    """sel_bias None is no key at all, and a pair of None is a norm of weight 1 and bias 0."""
    from test_gpu_routed import Layer
    d, E, T = 128, 8, 5
    x = torch.randn((T, d), generator=torch.Generator().manual_seed(3))
    with Layer(d, E, 8, True) as L:
        outs = []
        for norms, topk in (((None, None), dict(k=2, sel_bias=None)), ((None, None), dict(k=2)),
                            ((torch.ones(d).cuda(), torch.zeros(d).cuda()), dict(k=2))):
            st = DecodeStack([L.h], d, E, T, 0.5, norms=[norms], topk=topk)
            st.set_input(x)
            st.enqueue()
            torch.cuda.synchronize()
            outs.append(st.output.clone())
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        assert bool((outs[0].cpu() != x).any())
