"""GPU tests of single fp32 products in the routes that cut the factors into pieces: one k of each sum is not zero, so a result is one
product and nothing averages out."""
import math

import pytest
import torch

import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu

# Derived: what is left out of the nine products, 2^-24 (1 + 2^-10); the additions of the small products, below 2^-7 of the result,
# 5 * 2^-23 * 2^-7; the last addition, if it cuts off, 2^-23; one addition of parts, 2^-24.
BOUND = 2.0 ** -24 * (1 + 2.0 ** -10) + 5 * 2.0 ** -30 + 2.0 ** -23 + 2.0 ** -24


def factors(n, gen):
    """Numbers of [1, 2), among them those whose lower pieces are the largest."""
    bits = torch.randint(0, 1 << 23, (n,), generator=gen, device="cuda", dtype=torch.int32)
    worst = torch.tensor([0x00ffff, 0x0080ff, 0x007fff, 0x008000, 0x01ffff, 0x7fffff, 0x7f7fff, 0x017fff], dtype=torch.int32, device="cuda")
    bits[: min(n, 64)] = worst.repeat(8)[: min(n, 64)]
    sign = torch.randint(0, 2, (n,), generator=gen, device="cuda", dtype=torch.int32)
    return (bits | 0x3f800000).view(torch.float32) * (1 - 2 * sign)


def check(got, want, what):
    rel = ((got.double() - want) / want).abs().max().item()
    print("%s: 2^%.2f" % (what, math.log2(max(rel, 2.0 ** -60))), flush=True)
    assert rel <= BOUND, what


@pytest.mark.parametrize("M,N,K", [(4104, 2056, 200), (700, 300, 4000), (2500, 1365, 520), (600, 700, 2000)])
def test_one_product_is_exact_to_fp32(M, N, K):
    gen = torch.Generator(device="cuda").manual_seed(M)
    x, y = factors(M, gen), factors(N, gen)
    want = x.double()[:, None] * y.double()[None]
    for k in (0, K // 2, K - 1):
        a, w = torch.zeros(M, K, device="cuda"), torch.zeros(N, K, device="cuda")
        a[:, k], w[:, k] = x, y
        check(rcd.linear(a, w), want, "y")
        _, saved = rcd.gated_linear(a, w, w, act="none", want_saved=True)
        check(saved[..., 0], want, "g")
        check(saved[..., 1], want, "u")
    # the gradients: dA over N, dW over M
    p, q, r = factors(M, gen), factors(K, gen), factors(N, gen)
    dy, w = torch.zeros(M, N, device="cuda"), torch.zeros(N, K, device="cuda")
    dy[:, N - 1], w[N - 1] = p, q
    check(rcd.linear_backward(dy, torch.zeros(M, K, device="cuda"), w, want_dbias=False)[0], p.double()[:, None] * q.double()[None], "da")
    dy, a = torch.zeros(M, N, device="cuda"), torch.zeros(M, K, device="cuda")
    dy[M - 1], a[M - 1] = r, q
    check(rcd.linear_backward(dy, a, torch.zeros(N, K, device="cuda"), want_dbias=False)[1], r.double()[:, None] * q.double()[None], "dw")


def test_the_largest_numbers_stay_finite():
    """The nearest bf16 to the largest fp32 numbers is infinite; their pieces are not."""
    M, N, K = 4104, 2056, 200
    a, w = torch.zeros(M, K, device="cuda"), torch.zeros(N, K, device="cuda")
    largest = torch.finfo(torch.float32).max
    a[:, 5], w[:, 5] = largest, 1.0
    a[1::2, 5] = -largest
    got = rcd.linear(a, w)
    assert torch.equal(got[::2], torch.full_like(got[::2], largest)) and torch.equal(got[1::2], torch.full_like(got[1::2], -largest))
