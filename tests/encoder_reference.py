"""Plain 64-bit forms of the encoder's operators (torch on the CPU or the GPU, elementary operations only) and the error
bounds that the tests hold the kernels to.  The bounds are derived from the arithmetic, element by element:

  u = 2^-24 is fp32's unit roundoff (24 significant bits), w = 2^-8 bf16's (8 significant bits).  A sum of n products in fp32, in any order, is off by at most
  (n + 8) * 2u * sum |a||b| (the factor two allows accumulation that truncates).  An activation's value and slope have a
  Lipschitz constant below 1.2 and are themselves computed to 8u (1 + |z|).  Storing adds u or w relative.
"""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def unit(dtype):
    return U32 if dtype == torch.float32 else U16


def act_both(z, act):
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z), (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def act_error(z, ez, act):
    """Bounds on the errors of value and slope where z is off by up to ez."""
    if act == "none":
        return ez, torch.zeros_like(z)
    if act == "relu":
        return ez, (z.abs() <= ez).to(z.dtype)
    own = 8 * U32 * (1 + z.abs())
    return 1.2 * ez + own, 1.2 * ez + own


def sum_error(n, magnitude):
    return (n + 8) * 2 * U32 * magnitude


def mx_values(q, scale):
    """What 8-bit elements and scales stand for, in 64 bits."""
    e = scale.view(torch.uint8).double() - 127
    return q.double() * torch.pow(2.0, e).repeat_interleave(32, dim=1)[:, : q.shape[1]]


def norm(x, w, eps, r=None):
    h = x.double() if r is None else x.double() + r.double()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    y = h * rstd if w is None else h * rstd * w.double()
    return h, rstd, y


def norm_error(x, r, y, w, rstd, h, d):
    """Bound on y's error before it is stored: h is off by u |h|, rstd by (d + 16) u relative."""
    return (d + 24) * U32 * y.abs() + (0 if r is None else 2 * U32 * (h * rstd).abs() * (1 if w is None else w.double().abs()))


def linear(a, w, b, act, r):
    z = a @ w.t()
    if b is not None:
        z = z + b
    value, _ = act_both(z, act)
    return z, value if r is None else value + r


def linear_error(a, w, b, act, z):
    ez = sum_error(a.shape[1], a.abs() @ w.abs().t()) + (0 if b is None else U32 * z.abs())
    return ez, act_error(z, ez, act)[0]


def linear_backward(dy, a, w, z, act):
    dz = dy * act_both(z, act)[1]
    return dz, dz @ w, dz.t() @ a, dz.sum(0)


def gated(a, wg, wu, act):
    g, u = a @ wg.t(), a @ wu.t()
    return g, u, act_both(g, act)[0] * u


def gated_backward(dh, a, wg, wu, g, u, act):
    value, slope = act_both(g, act)
    dg, du = dh * u * slope, dh * value
    return dg, du, dg @ wg + du @ wu, dg.t() @ a, du.t() @ a
