"""Gradients of queries that see one key: its weight is 1 whatever the scores are, so q, k and the bias have a gradient of exactly zero there,
and the value's is the sum of dout.  A residue of rounding instead would be a full step to an optimiser that divides by the gradient's size."""
import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, forward_and_backward, generator, normal

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def zero(*tensors):
    for t in tensors:
        assert t is None or not bool(t.any()), t[t != 0].flatten()[:4]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 64), (3, 1, 6, 3, 40), (2, 5, 4, 1, 128), (1, 70, 2, 2, 65), (2, 130, 4, 2, 128), (60, 200, 4, 4, 64), (60, 200, 4, 4, 128)])
def test_one_key_in_all(size, causal, dtype):
    batch, n, heads, kv, d = size
    gen = generator(batch, n, d, causal, 31)
    q, dout = normal(gen, batch, n, heads, d, dtype=dtype, scale=3.0), normal(gen, batch, n, heads, d, dtype=dtype)
    k, v = normal(gen, batch, 1, kv, d, dtype=dtype), normal(gen, batch, 1, kv, d, dtype=dtype)
    for bias in (None, normal(gen, 12, heads, dtype=dtype)):
        _, _, grads = forward_and_backward(q, k, v, dout, ref.padded(batch, [1] * batch), bias, 40, causal=causal)
        zero(grads.dq, grads.dk, grads.dbias)
        assert bool(grads.dv.any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
def test_samples_of_one_token(causal, dtype):
    gen = generator(causal, 32)
    rows, heads, kv, d = 300, 4, 2, 48
    q, dout = normal(gen, rows, heads, d, dtype=dtype), normal(gen, rows, heads, d, dtype=dtype)
    k, v = normal(gen, rows, kv, d, dtype=dtype), normal(gen, rows, kv, d, dtype=dtype)
    bias = normal(gen, 16, heads, dtype=dtype)
    at = torch.arange(rows + 1, dtype=torch.int32, device=DEV)
    for b, longest in ((bias, 1), (None, 0), (bias, 300)):
        _, _, grads = forward_and_backward(q, k, v, dout, ref.ragged(list(range(rows + 1))), b, 40, causal=causal, q_offsets=at, k_offsets=at, longest_q=longest,
                                           longest_k=longest)
        zero(grads.dq, grads.dk, grads.dbias)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 33, 128])
def test_lengths_of_one_among_others(d, causal, dtype):
    """(The others' queries are cut into parts that are added up.)"""
    gen = generator(d, causal, 33)
    lengths, n, heads, kv = [1, 600, 1, 0], 600, 6, 2
    q, dout = normal(gen, 4, n, heads, d, dtype=dtype), normal(gen, 4, n, heads, d, dtype=dtype)
    k, v = normal(gen, 4, n, kv, d, dtype=dtype), normal(gen, 4, n, kv, d, dtype=dtype)
    at = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for bias in (None, normal(gen, 16, heads, dtype=dtype)):
        _, _, grads = forward_and_backward(q, k, v, dout, ref.padded(4, lengths), bias, 40, causal=causal, k_lengths=at)
        for b in (0, 2):
            zero(grads.dq[b], grads.dk[b])
        assert bool(grads.dq[1, -1].any()) and bool(grads.dk[1, 0].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 40, 40, 2, 2, 64), (2, 300, 300, 4, 2, 128), (2, 300, 300, 4, 2, 33), (30, 260, 260, 8, 8, 64), (30, 260, 260, 8, 8, 128),
                                  (2, 90, 60, 2, 1, 72)])
def test_the_first_query_of_a_causal_call(size, dtype):
    batch, n, m, heads, kv, d = size
    gen = generator(n, m, d, 34)
    q, k, v = normal(gen, batch, n, heads, d, dtype=dtype), normal(gen, batch, m, kv, d, dtype=dtype), normal(gen, batch, m, kv, d, dtype=dtype)
    dout = normal(gen, batch, n, heads, d, dtype=dtype)
    first = n - m                       # the query at position 0
    alone = torch.zeros_like(dout)
    alone[:, :first + 1] = dout[:, :first + 1]
    for bias in (None, normal(gen, 16, heads, dtype=dtype)):
        _, _, grads = forward_and_backward(q, k, v, dout, ref.padded(batch, [m] * batch), bias, 40, causal=True)
        zero(grads.dq[:, :first + 1])
        assert bool(grads.dq[:, first + 1].any()) and bool(grads.dk[:, 0].any())
        # nothing but that query's gradient: it goes to the first value and nowhere else
        _, _, grads = forward_and_backward(q, k, v, alone, ref.padded(batch, [m] * batch), bias, 40, causal=True)
        zero(grads.dq, grads.dk, grads.dbias, grads.dv[:, 1:])
        assert bool(grads.dv[:, 0].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [30, 200])
def test_beside_what_is_not_finite(n, dtype):
    """A key and a query of NaN further on: their tiles are added up row by row."""
    gen = generator(n, 35)
    q, k, v, dout = (normal(gen, 1, n, 2, 64, dtype=dtype) for _ in range(4))
    bad = 20
    k2, q2, dout2 = k.clone(), q.clone(), dout.clone()
    k2[:, bad] = float("nan")
    out, saved = rcd.attention(q, k2, v, causal=True, want_saved=True)
    zero(rcd.attention_backward(dout, q, k2, v, out, saved, causal=True).dq[:, 0])
    q2[:, bad], dout2[:, bad] = float("nan"), float("inf")
    dout2[:, 1:bad] = 0
    dout2[:, bad + 1:] = 0
    out, saved = rcd.attention(q2, k, v, causal=True, want_saved=True)
    grads = rcd.attention_backward(dout2, q2, k, v, out, saved, causal=True)
    zero(grads.dq[:, :bad], grads.dq[:, bad + 1:], grads.dk[:, bad + 1:], grads.dv[:, bad + 1:])
