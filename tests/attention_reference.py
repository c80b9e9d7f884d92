"""Attention and its gradients from the definition in 64 bits, and how far off a kernel may be that rounds as it says it does.

What rounds, with h = half a step of the type (bf16 2^-8, fp32 2^-24) and u = 2^-24:
  a score        sums of d products in fp32: (d + 4) u sum |q k| scale, the bias and the exponent's argument: 4 u (|s| + |largest s|)
  p              twice that relative, plus its row's sum and the powers of two: (keys + 32) u; in bf16 h on its way into the product
  out            h
  dp             (d + 4) u sum |dout v|;  delta: the same, and h sum |dout out|, since out is taken as it left
  ds             p times those, plus p's own error; in bf16 h on its way into the product
  dq, dk, dv     (terms + 4) u of the sum of the terms' sizes, and h
"""
import math

import torch

U = 2.0 ** -24


def bucket_table(buckets, distance, causal):
    """Bucket of each distance up to `distance`, by whole powers."""
    n = buckets if causal else buckets // 2
    half = n // 2
    table = []
    for r in range(distance + 1):
        if r < half:
            table.append(r)
            continue
        c = 0
        while c < n - half - 1 and r ** (n - half) * half ** (c + 1) >= half ** (n - half) * distance ** (c + 1):
            c += 1
        table.append(half + c)
    return table


def buckets_of(offset, buckets, distance, causal):
    table = torch.tensor(bucket_table(buckets, distance, causal), device=offset.device)
    b = table[offset.abs().clamp(max=distance)]
    return b if causal else b + (offset > 0) * (buckets // 2)


def one_head(q, k, v, scale, causal, bias=None, bucket=None, dout=None, half=U, rounds=False):
    """({name: value}, {name: bound}) of one head of one sequence; half: h of the type, rounds: p and ds pass through it."""
    w = torch.float64
    q, k, v = q.to(w), k.to(w), v.to(w)
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    seen = torch.ones(n, m, dtype=torch.bool, device=q.device)
    if causal:
        seen = torch.arange(m, device=q.device)[None, :] <= (torch.arange(n, device=q.device) + (m - n))[:, None]
    score = q @ k.t() * scale
    size = q.abs() @ k.abs().t() * scale
    if bias is not None:
        score = score + bias.to(w)[bucket]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(1, keepdim=True) if m else torch.full((n, 1), -math.inf, dtype=w, device=q.device)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score - top)
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    finite = torch.where(torch.isfinite(score), score.abs(), 0.0)
    off = (d + 4) * U * size + 4 * U * (finite + (finite.amax(1, keepdim=True) if m else 0))
    off = torch.where(seen, off, 0.0)
    rel = off + (off.amax(1, keepdim=True) if m else 0) + (m + 32) * U
    dp_in = half if rounds else 0.0
    out = p @ v
    value = {"out": out}
    bound = {"out": (p * (rel + dp_in)) @ v.abs() + (m + 4) * U * (p @ v.abs()) + half * out.abs() + 1e-30}
    if dout is None:
        return value, bound
    g = dout.to(w)
    delta = (g * out).sum(1, keepdim=True)
    dp = g @ v.t()
    ds = p * (dp - delta)
    value["dv"] = p.t() @ g
    bound["dv"] = (p * (rel + dp_in + (n + 4) * U)).t() @ g.abs() + half * value["dv"].abs() + 1e-30
    e_delta = (d + 4) * U * (g.abs() * out.abs()).sum(1, keepdim=True) + (g.abs() * (bound["out"])).sum(1, keepdim=True)
    e_dp = (d + 4) * U * (g.abs() @ v.abs().t())
    e_ds = p * (e_dp + e_delta) + ds.abs() * (rel + 4 * U)
    for name, x, t, terms in (("dq", k, ds, m), ("dk", q, ds.t(), n)):
        e_x = (e_ds if name == "dq" else e_ds.t()) + (dp_in + (terms + 4) * U) * t.abs()
        value[name] = t @ x * scale
        bound[name] = e_x @ x.abs() * scale + half * value[name].abs() + 1e-30
    if bias is not None:
        flat = bucket.reshape(-1)
        for name, t in (("value", ds), ("bound", e_ds + (n * m + 64) * U * ds.abs() if n * m < 64 else e_ds + 256 * U * ds.abs())):
            into = torch.zeros(bias.shape[0], dtype=w, device=q.device).index_add_(0, flat, t.reshape(-1))
            (value if name == "value" else bound)["dbias"] = into
    return value, bound


def attention(q, k, v, scale=None, causal=False, sequences=None, bias=None, distance=128, dout=None):
    """values and bounds of whole tensors.  sequences: [(index of q's rows, index of k's rows)] into the tensors; rows in none of
    them have value 0 and bound 0."""
    half = torch.finfo(q.dtype).eps / 2
    rounds = q.dtype == torch.bfloat16
    scale = float(torch.tensor(q.shape[-1] ** -0.5 if scale is None else scale, dtype=torch.float32))
    H, group = q.shape[-2], q.shape[-2] // k.shape[-2]
    names = {"out": q} if dout is None else {"out": q, "dq": q, "dk": k, "dv": v}
    value = {n: torch.zeros(t.shape, dtype=torch.float64, device=q.device) for n, t in names.items()}
    bound = {n: torch.zeros_like(t) for n, t in value.items()}
    if dout is not None and bias is not None:
        value["dbias"] = torch.zeros(bias.shape, dtype=torch.float64, device=q.device)
        bound["dbias"] = torch.zeros_like(value["dbias"])
    for iq, ik in sequences:
        n, m = q[iq].shape[0], k[ik].shape[0]
        bucket = None
        if bias is not None:
            offset = torch.arange(m, device=q.device)[None, :] - (torch.arange(n, device=q.device) + (m - n))[:, None]
            bucket = buckets_of(offset, bias.shape[0], distance, causal)
        for h in range(H):
            a, b = one_head(q[iq][:, h], k[ik][:, h // group], v[ik][:, h // group], scale, causal, None if bias is None else bias[:, h], bucket,
                            None if dout is None else dout[iq][:, h], half, rounds)
            for name in a:
                for into, part in ((value, a), (bound, b)):
                    if name in ("out", "dq"):
                        into[name][iq][:, h] = part[name]
                    elif name in ("dk", "dv"):
                        into[name][ik][:, h // group] += part[name]
                    else:
                        into[name][:, h] += part[name]
    if "dbias" in value:
        bound["dbias"] += torch.finfo(bias.dtype).eps / 2 * value["dbias"].abs() + 1e-30
    return value, bound


def ragged(offsets):
    """The sequences of two equal lists of offsets."""
    return [(slice(a, b), slice(a, b)) for a, b in zip(offsets[:-1], offsets[1:])]


def padded(batch, lengths):
    return [((b, slice(None)), (b, slice(0, n))) for b, n in zip(range(batch), lengths)]


def check(name, got, value, bound):
    assert got.shape == value.shape, (name, got.shape, value.shape)
    got = got.to(torch.float64)
    bad = ~((got - value).abs() <= bound)
    if bool(bad.any()):
        at = torch.nonzero(bad)[0].tolist()
        raise AssertionError("%s: %d of %d off, first at %s: %r, wanted %r within %r" % (
            name, int(bad.sum()), bad.numel(), at, got[tuple(at)].item(), value[tuple(at)].item(), bound[tuple(at)].item()))
