"""GPU tests of the encoder's calls beside autograd: what requires grad is refused while gradients are recorded, whichever argument it
is; inside an autograd.Function the calls carry gradients; a result written into a tensor counts as a change of it."""
import pytest
import torch

import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu

UNSUPPORTED = 4


def make(*shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(sum(shape)), device="cuda")


def arguments():
    M, N, K = 20, 12, 16
    a, w, dy = make(M, K), make(N, K), make(M, N)
    rstd = rcd.rms_norm(a, want_rstd=True).rstd
    _, z = rcd.linear(a, w, want_preact=True)
    _, saved = rcd.gated_linear(a, w, w, want_saved=True)
    return [(rcd.rms_norm, dict(x=a, weight=make(K), residual=make(M, K))),
            (rcd.rms_norm_backward, dict(dy=make(M, K), h=a, rstd=rstd, weight=make(K), dsum=make(M, K))),
            (rcd.quantize_mxfp8, dict(x=a)),
            (rcd.linear, dict(a=a, w=w, bias=make(N), residual=make(M, N), out=torch.empty(M, N, device="cuda"))),
            (rcd.linear_backward, dict(dy=dy, a=a, w=w, preact=z, act="silu")),
            (rcd.gated_linear, dict(a=a, w_gate=w, w_up=make(N, K) + 1, out=torch.empty(M, N, device="cuda"))),
            (rcd.gated_linear_backward, dict(dh=dy, a=a, w_gate=w, w_up=make(N, K) + 1, saved=saved))]


def test_whichever_argument_requires_grad_is_refused_while_gradients_are_recorded():
    for call, given in arguments():
        call(**given)
        for name, t in given.items():
            if not isinstance(t, torch.Tensor):
                continue
            spoilt = dict(given, **{name: t.clone().requires_grad_(True)})
            with pytest.raises(rcd.RcdError) as e:
                call(**spoilt)
            assert e.value.status == UNSUPPORTED and "grad" in str(e.value), (call.__name__, name)
            with torch.no_grad():
                call(**spoilt)


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, a, w):
        y, z = rcd.linear(a, w, act="silu", want_preact=True)
        ctx.save_for_backward(a, w, z)
        return y

    @staticmethod
    def backward(ctx, dy):
        a, w, z = ctx.saved_tensors
        return rcd.linear_backward(dy, a, w, z, act="silu", want_dbias=False)[:2]


def test_an_autograd_function_carries_gradients():
    a, w = make(20, 16).requires_grad_(True), make(12, 16).requires_grad_(True)
    Linear.apply(a, w).square().sum().backward()
    a2, w2 = a.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
    torch.nn.functional.silu(a2 @ w2.t()).square().sum().backward()
    for got, want in ((a.grad, a2.grad), (w.grad, w2.grad)):
        assert (got.double() - want).norm() <= 1e-5 * want.norm()


def test_a_result_written_into_a_tensor_counts_as_a_change_of_it():
    a, w = make(20, 16), make(12, 16)
    out = torch.zeros(20, 12, device="cuda")
    before = out._version
    rcd.linear(a, w, out=out)
    rcd.gated_linear(a, w, w, out=out)
    assert out._version == before + 2
    # so autograd notices that what it has kept is gone
    x = torch.ones(20, 12, device="cuda", requires_grad=True)
    y = x * out
    with torch.no_grad():
        rcd.linear(a, w, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with torch.inference_mode():
        kept = torch.empty(20, 12, device="cuda")
        assert rcd.linear(a, w, out=kept) is kept and torch.equal(kept, rcd.linear(a, w))
