"""GPU test of the way from hidden states to a partition (examples/encode_and_partition.py): training lowers the error, the
gradients are the loss's, 8-bit features stay near the bf16 ones, and the partition has the quotas of its capacities."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2211_00839_amd as rcd

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import encode_and_partition as example  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
def test_hidden_states_to_partition(bits):
    got = example.run(samples=3001, width=200, inner=333, features=48, classes=4, layers=2, steps=40, batch=1024, bits=bits)
    assert np.mean(got["losses"][-5:]) < 0.5 * got["losses"][0]
    assert torch.all(torch.isfinite(got["features"].float()))
    assert (got["features"].float() - got["plain"].float()).norm() <= 0.15 * got["plain"].float().norm()
    labels, assign = got["labels"].cpu().numpy(), got["assign"].cpu().numpy()
    for c in range(4):
        want = oracle.quota(int((labels == c).sum()), np.array([1, 1, 2, 4], dtype=np.int32))
        assert [int(((labels == c) & (assign == k)).sum()) for k in range(4)] == want.tolist()


def test_its_gradients_are_the_losss():
    """Against torch's own differentiation of the same layers in 64 bits on the CPU."""
    x, _ = example.make_hidden_states(257, 96, 3, 5)
    model = example.Encoder(96, 136, 24, 2, 6)
    loss, grad = model.loss_and_gradients(x)
    p = {k: v.double().cpu().requires_grad_(True) for k, v in model.p.items()}

    def norm(h, w):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + example.EPS) * w

    r = xd = x.double().cpu()
    for i in range(2):
        n = norm(r, p["scale%d" % i])
        g, u = n @ p["gate%d" % i].t(), n @ p["up%d" % i].t()
        r = r + (g / (1 + torch.exp(-g)) * u) @ p["down%d" % i].t()
    f = norm(r, p["scale"]) @ p["head"].t() + p["head_bias"]
    off = f @ p["back"].t() + p["back_bias"] - xd
    assert abs(loss.item() - off.square().mean().item()) <= 0.02 * loss.item()
    (off.square().sum() / off.shape[0]).backward()
    for k, g in grad.items():
        want = p[k].grad
        # some twenty roundings to bf16 (2^-9 on average, independent) lie between the input and the first layer's gradients
        assert (g.double().cpu() - want).norm() <= 0.03 * want.norm(), k
