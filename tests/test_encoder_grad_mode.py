"""CPU tests: a tensor whose gradients autograd is expected to record is refused, whichever argument it is, before anything else
about it is looked at; with recording off it is taken like any other (and then refused for not being on a device)."""
import pytest
import torch

import paper_2211_00839_amd as rcd

UNSUPPORTED, NOT_ON_DEVICE = 4, -1


def status(call, *args, **kwargs):
    with pytest.raises(rcd.RcdError) as e:
        call(*args, **kwargs)
    return e.value.status


def leaf(*shape):
    return torch.zeros(*shape, requires_grad=True)


CALLS = [(rcd.rms_norm, (4, 8)), (rcd.quantize_mxfp8, (4, 8)), (rcd.linear, (4, 8), (6, 8)), (rcd.gated_linear, (4, 8), (6, 8), (6, 8)),
         (rcd.linear_backward, (4, 6), (4, 8), (6, 8)), (rcd.rms_norm_backward, (4, 8), (4, 8), (4,)),
         (rcd.gated_linear_backward, (4, 6), (4, 8), (6, 8), (6, 8), (4, 6, 2))]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c[0].__name__)
def test_the_first_argument(call):
    f, first, *others = call
    others = [torch.zeros(*shape) for shape in others]
    assert status(f, leaf(*first), *others) == UNSUPPORTED
    assert status(f, leaf(*first).detach(), *others) == NOT_ON_DEVICE
    with torch.no_grad():
        assert status(f, leaf(*first), *others) == NOT_ON_DEVICE
    with torch.inference_mode():
        assert status(f, leaf(*first), *others) == NOT_ON_DEVICE
