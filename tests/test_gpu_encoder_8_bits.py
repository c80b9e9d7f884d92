"""GPU tests of how exact the sums of 8-bit products are, around the length and the numbers of rows at which they go another way.

The bounds, derived before any run.  A product of two 8-bit values has at most 8 significant bits, so in an fp32 sum only the
additions round, each by up to 2^-24 of the partial sum.  With products of random signs the partial sums are a random walk of
rms size sqrt(k / K) s, s = sqrt(sum p^2), and the K errors (rms 2^-24 / sqrt 3 of the partial sum each) are independent: their sum
has an rms below sqrt(K) 2^-24 s / sqrt 6.  The tests allow sqrt(K) 2^-24 s.  With products of one sign the partial sums grow to
P = sum |p|, an output's error has an rms below sqrt(K) 2^-24 P / 3, and its mean over many outputs is near zero: they allow a
quarter of sqrt(K) 2^-24 P for the mean, which an accumulation that always cuts towards the same side would pass.
"""
import math

import pytest
import torch

import encoder_reference as ref
import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def operands(kind, rows, N, K):
    gen = torch.Generator(device="cuda").manual_seed(K)
    x, w = torch.randn(rows, K, generator=gen, device="cuda"), torch.randn(N, K, generator=gen, device="cuda")
    if kind == "outliers":
        x[:, ::64] *= 10
    elif kind == "one sign":
        x, w = x.abs(), w.abs()
    elif kind == "cancelling":      # the second half of each sum takes most of the first away
        half = K // 2
        w[:, half: 2 * half] = -w[:, :half]
        x[:, half: 2 * half] = x[:, :half] * (1 + 0.01 * torch.randn(rows, half, generator=gen, device="cuda"))
    return rcd.quantize_mxfp8(x), rcd.quantize_mxfp8(w)


def check_sums(got, a, w, kind, what):
    K = a.shape[1]
    err = got.double() - a @ w.t()
    if kind == "one sign":
        size = (a.abs() @ w.abs().t()).mean().item()
        off, allowed = abs(err.mean().item()), math.sqrt(K) * 2.0 ** -26 * size
    else:
        size = (a.square() @ w.square().t()).mean().sqrt().item()
        off, allowed = err.square().mean().sqrt().item(), math.sqrt(K) * 2.0 ** -24 * size
    print("%s: %.3f of the bound" % (what, off / allowed), flush=True)
    assert off <= allowed, what


@pytest.mark.parametrize("kind", ["random", "outliers", "one sign", "cancelling"])
@pytest.mark.parametrize("K", [2047, 2048, 8192])
def test_sums_that_leave_in_fp32_are_fp32_sums(K, kind):
    (a, sa), (w, sw) = operands(kind, 300, 200, K)
    ad, wd = ref.mx_values(a, sa), ref.mx_values(w, sw)
    for M in (16, 17, 33, 65, 300):
        what = "%s, K %d, %d rows" % (kind, K, M)
        check_sums(rcd.linear(a[:M], w, a_scale=sa[:M], w_scale=sw, out_dtype=F32), ad[:M], wd, kind, what)
        _, z = rcd.linear(a[:M], w, a_scale=sa[:M], w_scale=sw, want_preact=True)
        check_sums(z, ad[:M], wd, kind, what + ", z beside a bf16 result")
        for out_dtype in (F32, BF16):
            _, saved = rcd.gated_linear(a[:M], w, w, a_scale=sa[:M], gate_scale=sw, up_scale=sw, out_dtype=out_dtype, want_saved=True)
            check_sums(saved[..., 0], ad[:M], wd, kind, what + ", g")
            check_sums(saved[..., 1], ad[:M], wd, kind, what + ", u")
        h = rcd.gated_linear(a[:M], w, w, act="relu", a_scale=sa[:M], gate_scale=sw, up_scale=sw, out_dtype=F32)
        same, _ = rcd.gated_linear(a[:M], w, w, act="relu", a_scale=sa[:M], gate_scale=sw, up_scale=sw, out_dtype=F32, want_saved=True)
        assert torch.equal(h, same)


@pytest.mark.parametrize("kind", ["random", "outliers", "one sign"])
@pytest.mark.parametrize("K", [2047, 2048, 8192])
def test_bf16_results_are_off_by_little_more_than_their_rounding(K, kind):
    """Of each result: its rounding, and at most 2^-12 of its products' sizes.  In the mean (rms): within a twentieth of the
    rounding alone, at every number of rows."""
    (a, sa), (w, sw) = operands(kind, 300, 200, K)
    ad, wd = ref.mx_values(a, sa), ref.mx_values(w, sw)
    for M in (16, 17, 33, 65, 300):
        want, size = ad[:M] @ wd.t(), ad[:M].abs() @ wd.abs().t()
        off = rcd.linear(a[:M], w, a_scale=sa[:M], w_scale=sw).double() - want
        assert torch.all(off.abs() <= ref.U16 * want.abs() + 2.0 ** -12 * size)
        rounding = (want.bfloat16().double() - want).norm()
        assert off.norm() <= 1.05 * rounding, (M, (off.norm() / rounding).item())


def test_a_given_workspace_is_enough_for_either_result():
    M, N, K = 300, 200, 2048
    (a, sa), (w, sw) = operands("random", M, N, K)
    lib = rcd.load_library()
    for query, call in ((lib.rcd_linear_workspace_bytes, lambda t, ws: rcd.linear(a, w, a_scale=sa, w_scale=sw, out_dtype=t, workspace=ws)),
                        (lib.rcd_gated_linear_workspace_bytes,
                         lambda t, ws: rcd.gated_linear(a, w, w, a_scale=sa, gate_scale=sw, up_scale=sw, out_dtype=t, workspace=ws))):
        need = query(M, N, K, rcd.MXFP8)
        for t in (F32, BF16):
            ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")      # NaN wherever it is read before it is written
            assert torch.equal(call(t, ws[:need]), call(t, None)) and torch.all(ws[need:] == 0xff)
