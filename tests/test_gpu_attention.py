"""Attention and its gradients against the definition in 64 bits, with what the roundings allow."""
import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu

DEV = "cuda"


def normal(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(dtype)


def generator(*of):
    return torch.Generator(device=DEV).manual_seed(sum(int(x) * 7919 ** i for i, x in enumerate(of)) % 2 ** 31)


def forward_and_backward(q, k, v, dout, sequences, bias=None, distance=128, **how):
    """Runs both calls and compares everything."""
    kwargs = dict(how, bias=bias, max_distance=distance)
    out, saved = rcd.attention(q, k, v, want_saved=True, **kwargs)
    again = rcd.attention(q, k, v, **kwargs)
    assert torch.equal(out.view(torch.uint8), again.view(torch.uint8))
    grads = rcd.attention_backward(dout, q, k, v, out, saved, **kwargs)
    value, bound = ref.attention(q, k, v, how.get("scale"), how.get("causal", False), sequences, bias, distance, dout)
    for name, got in (("out", out), ("dq", grads.dq), ("dk", grads.dk), ("dv", grads.dv), ("dbias", grads.dbias)):
        if got is not None:
            ref.check(name, got, value[name], bound[name])
    return out, saved, grads


# (queries, keys), (heads, kv_heads), d
SIZES = [(1, 1, 1, 1, 1), (1, 7, 2, 1, 64), (5, 33, 3, 3, 40), (31, 32, 2, 2, 128), (32, 31, 4, 2, 17), (33, 65, 2, 2, 64), (64, 64, 6, 2, 96),
         (65, 129, 2, 2, 128), (128, 128, 2, 1, 64), (129, 100, 2, 2, 65), (200, 300, 4, 4, 8), (300, 300, 3, 1, 120), (257, 513, 2, 2, 64),
         (7, 1100, 8, 2, 128), (1, 2500, 4, 4, 72)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_dense(size, causal, dtype):
    n, m, heads, kv, d = size
    gen = generator(n, m, d, causal)
    q, dout = normal(gen, 2, n, heads, d, dtype=dtype, scale=2.0), normal(gen, 2, n, heads, d, dtype=dtype)
    k, v = normal(gen, 2, m, kv, d, dtype=dtype), normal(gen, 2, m, kv, d, dtype=dtype)
    forward_and_backward(q, k, v, dout, ref.padded(2, [m, m]), causal=causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_bias(size, causal, dtype):
    n, m, heads, kv, d = size
    gen = generator(n, m, d, causal, 1)
    q, dout = normal(gen, 2, n, heads, d, dtype=dtype), normal(gen, 2, n, heads, d, dtype=dtype)
    k, v = normal(gen, 2, m, kv, d, dtype=dtype), normal(gen, 2, m, kv, d, dtype=dtype)
    for buckets, distance, type_ in ((12, 50, dtype), (4, 3, torch.float32), (32, 128, dtype), (64, 600, torch.float32)):
        bias = normal(gen, buckets, heads, dtype=type_, scale=2.0)
        forward_and_backward(q, k, v, dout, ref.padded(2, [m, m]), bias, distance, causal=causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 33, 128])
def test_ragged(d, causal, dtype):
    """Sequences of no and of one token among them, rows in front and behind that belong to none, views of one projection."""
    gen = generator(d, causal, 2)
    offsets = [3, 3, 4, 37, 37, 165, 294, 300, 555]
    rows = 560
    qkv = normal(gen, rows, 8, d, dtype=dtype)
    q, k, v = qkv.split([4, 2, 2], dim=1)
    dout = normal(gen, rows, 4, d, dtype=dtype)
    bias = normal(gen, 16, 4, dtype=dtype)
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    for longest in (0, 255, 1):
        for b in (None, bias):
            forward_and_backward(q, k, v, dout, ref.ragged(offsets), b, 40, causal=causal, q_offsets=at, k_offsets=at, longest_q=longest, longest_k=longest)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(causal, dtype):
    """Keys behind each sequence's length are NaN; some sequences have none, some queries see nothing."""
    gen = generator(causal, 3)
    lengths = [0, 1, 40, 64, 129, 200, 77]
    B, n, m, heads, kv, d = len(lengths), 70, 200, 4, 2, 64
    q, dout = normal(gen, B, n, heads, d, dtype=dtype), normal(gen, B, n, heads, d, dtype=dtype)
    k, v = normal(gen, B, m, kv, d, dtype=dtype), normal(gen, B, m, kv, d, dtype=dtype)
    for b, length in enumerate(lengths):
        k[b, length:] = float("nan")
        v[b, length:] = float("inf")
    at = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    bias = normal(gen, 16, heads, dtype=dtype)
    for x in (None, bias):
        forward_and_backward(q, k, v, dout, ref.padded(B, lengths), x, 40, causal=causal, k_lengths=at)
        out = rcd.attention(q[:, :3], k, v, causal=causal, k_lengths=at, bias=x, max_distance=40)
        value, bound = ref.attention(q[:, :3], k, v, None, causal, ref.padded(B, lengths), x, 40)
        ref.check("out", out, value["out"], bound["out"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ragged_queries_over_a_cache(dtype):
    gen = generator(4)
    offsets, lengths = [0, 5, 5, 6, 40], [300, 20, 1, 130]
    heads, kv, d = 4, 1, 128
    q, dout = normal(gen, 40, heads, d, dtype=dtype), normal(gen, 40, heads, d, dtype=dtype)
    k, v = normal(gen, 4, 320, kv, d, dtype=dtype), normal(gen, 4, 320, kv, d, dtype=dtype)
    sequences = [(slice(a, b), (i, slice(0, n))) for i, (a, b, n) in enumerate(zip(offsets[:-1], offsets[1:], lengths))]
    for causal in (False, True):
        forward_and_backward(q, k, v, dout, sequences, None, 128, causal=causal, q_offsets=torch.tensor(offsets, dtype=torch.int32, device=DEV),
                             k_lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 33, 128])
@pytest.mark.parametrize("n", [30, 200])
def test_nothing_comes_from_what_is_not_seen(n, d, dtype):
    """Causal: a key and value of NaN and infinities reaches no query in front of it, a query and gradient of them no key behind it."""
    gen = generator(n, d, 5)
    heads, kv, bad = 4, 2, n - 20
    q, dout = normal(gen, 1, n, heads, d, dtype=dtype), normal(gen, 1, n, heads, d, dtype=dtype)
    k, v = normal(gen, 1, n, kv, d, dtype=dtype), normal(gen, 1, n, kv, d, dtype=dtype)
    value, bound = ref.attention(q, k, v, None, True, ref.padded(1, [n]), None, 128, dout)
    for bias in (None, torch.zeros(8, heads, device=DEV)):
        for fill in (float("nan"), float("inf")):
            k2, v2 = k.clone(), v.clone()
            k2[:, bad], v2[:, bad, :, ::2] = fill, fill
            out, saved = rcd.attention(q, k2, v2, causal=True, bias=bias, want_saved=True)
            grads = rcd.attention_backward(dout, q, k2, v2, out, saved, causal=True, bias=bias)
            ref.check("out", out[:, :bad], value["out"][:, :bad], bound["out"][:, :bad])
            ref.check("dq", grads.dq[:, :bad], value["dq"][:, :bad], bound["dq"][:, :bad])
            # an infinite value alone: where it stands, and in every query that sees it
            v3 = v.clone()
            v3[:, bad, :, 0] = fill
            out = rcd.attention(q, k, v3, causal=True, bias=bias)
            assert not out[:, bad:, :, 0].isfinite().any()
            ref.check("out", out[:, :bad], value["out"][:, :bad], bound["out"][:, :bad])
            ref.check("out", out[:, :, :, 1:], value["out"][:, :, :, 1:], bound["out"][:, :, :, 1:])
            q2, dout2 = q.clone(), dout.clone()
            q2[:, bad, :, 1::2], dout2[:, bad] = fill, fill
            out, saved = rcd.attention(q2, k, v, causal=True, bias=bias, want_saved=True)
            grads = rcd.attention_backward(dout2, q2, k, v, out, saved, causal=True, bias=bias)
            rest = [i for i in range(n) if i != bad]
            ref.check("out", out[:, rest], value["out"][:, rest], bound["out"][:, rest])
            ref.check("dq", grads.dq[:, rest], value["dq"][:, rest], bound["dq"][:, rest])
            for name in ("dk", "dv"):
                ref.check(name, getattr(grads, name)[:, bad + 1:], value[name][:, bad + 1:], bound[name][:, bad + 1:])
