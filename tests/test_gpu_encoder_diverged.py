"""GPU tests of fp32 products by pieces on what a diverged training step holds: NaN, infinities and sums past the largest number,
in a few places or everywhere.  They are what the formula makes of them in every route, and take no more than a small multiple of
a finite call."""
import time

import pytest
import torch

import encoder_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_encoder import F32, check, normal

pytestmark = pytest.mark.gpu

# large tiles and small ones, whole and in parts, both gradients side by side and one after the other
SIZES = [(4104, 2056, 200), (600, 700, 2000), (700, 300, 4000), (2500, 1365, 520), (200, 4104, 2056)]


def spoil(t, how):
    """A copy of t (rows x columns) with what `how` names put into it."""
    t = t.clone()
    if how == "a row of NaN":
        t[t.shape[0] // 2] = float("nan")
    elif how == "a column of NaN":
        t[:, -1] = float("nan")
    elif how == "an infinite column":
        t[:, 3] = float("inf")
    elif how == "opposite infinities":
        t[:, 3], t[:, 70] = float("inf"), float("-inf")
    elif how == "all NaN":
        t[:] = float("nan")
    elif how == "past the largest":
        t = (t.abs() + 0.5) * 1e25
    return t


HOWS = ["a row of NaN", "a column of NaN", "an infinite column", "opposite infinities", "all NaN", "past the largest"]


def product(a, w):
    """a w^T in 64 bits with fp32's range, and the bound of its finite elements."""
    y = a.double() @ w.double().t()
    y = torch.where(y.abs() > 3.5e38, torch.copysign(torch.full_like(y, float("inf")), y), y)
    clean = [torch.nan_to_num(t.double(), 0, 0, 0) for t in (a, w)]
    return y, ref.sum_error(a.shape[1], clean[0].abs() @ clean[1].abs().t())


@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_results_are_the_formulas(M, N, K, how):
    gen = torch.Generator(device="cuda").manual_seed(M + N)
    a, w = spoil(normal(gen, M, K), how), normal(gen, N, K, scale=K ** -0.5)
    w[5] = 0.5                       # exactly representable: its lower pieces are zero
    w[6] = 0.0                       # an infinity times zero
    if how == "past the largest":
        w = (w.abs() + 0.5) * 1e25
    y, bound = product(a, w)
    check(rcd.linear(a, w), y, bound, F32, "y")
    other = w.flip(0).contiguous()
    h, saved = rcd.gated_linear(a, w, other, act="none", want_saved=True)
    check(saved[..., 0], y, bound, F32, "g")
    check(saved[..., 1], y.flip(1), bound.flip(1), F32, "u")
    # gradients: the spoilt matrix is dy, then a
    dy, ok = spoil(normal(gen, M, N), how), normal(gen, M, K)
    da, dw, _ = rcd.linear_backward(dy, ok, w, want_dbias=False)
    check(da, *product(dy, w.t()), F32, "da")
    check(dw, *product(dy.t(), ok.t()), F32, "dw")
    assert torch.equal(torch.nan_to_num(rcd.linear_backward(dy, ok, w, want_da=False, want_dbias=False)[1], 1e9, 2e9, -2e9),
                       torch.nan_to_num(dw, 1e9, 2e9, -2e9))
    dy = normal(gen, M, N)
    _, dw, _ = rcd.linear_backward(dy, a, w, want_da=False, want_dbias=False)
    check(dw, *product(dy.t(), a.t()), F32, "dw of a spoilt input")
    # the gated block's weights: two gradients in one product
    saved = torch.ones(M, N, 2, device="cuda")
    da, dg, du = rcd.gated_linear_backward(dy, a, w, other, saved, act="none")
    want, bound = product(dy.t(), a.t())
    check(dg, want, bound, F32, "dw_gate")
    check(du, want, bound, F32, "dw_up")


def fastest(call):
    call()
    torch.cuda.synchronize()
    best = float("inf")
    for _ in range(3):
        t = time.perf_counter()
        call()
        torch.cuda.synchronize()
        best = min(best, time.perf_counter() - t)
    return best


@pytest.mark.parametrize("how", HOWS)
def test_a_diverged_step_takes_a_small_multiple_of_a_finite_one(how):
    """Of every call, whatever of its sums is not finite: at most forty times as long (one thread to a sum, which then walks all of k by
    itself, would take hundreds of times as long)."""
    M, N, K = 4104, 2056, 1040
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, w, dy = normal(gen, M, K), normal(gen, N, K), normal(gen, M, N)
    w = w.abs() + 0.5
    saved = torch.ones(M, N, 2, device="cuda")

    def calls(a, w, dy):
        return {"linear": lambda: rcd.linear(a, w), "linear_backward": lambda: rcd.linear_backward(dy, a, w),
                "gated_linear": lambda: rcd.gated_linear(a, w, w),
                "gated_linear_backward": lambda: rcd.gated_linear_backward(dy, a, w, w, saved)}

    finite = calls(a, w, dy)
    spoilt = calls(spoil(a, how), w * 1e25 if how == "past the largest" else w, spoil(dy, how))
    for name in finite:
        before = fastest(finite[name])
        now = fastest(spoilt[name])
        print("%s, %s: %.0f us, %.0f finite" % (name, how, now * 1e6, before * 1e6), flush=True)
        assert now <= 40 * before, name
