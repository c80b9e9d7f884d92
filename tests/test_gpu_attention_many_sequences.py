"""More sequences than a workgroup has threads, which finds its tile among them by rounds of as many: the counts carry over from round to round."""
import random

import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, forward_and_backward, generator, normal

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def offsets_of(lengths):
    offsets = [2]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    return offsets


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kind", ["short", "mixed", "empty first", "one at the end"])
def test_by_offsets(kind, causal, dtype):
    rng = random.Random(kind)
    count = 1300
    lengths = {"short": [rng.randint(0, 3) for _ in range(count)],
               "mixed": [rng.choice([0, 1, 2, 5, 33]) if rng.random() < 0.99 else rng.choice([130, 300]) for _ in range(count)],
               "empty first": [0] * 1100 + [rng.choice([1, 4, 40]) for _ in range(200)],
               "one at the end": [0] * (count - 1) + [200]}[kind]
    offsets = offsets_of(lengths)
    rows, heads, kv, d = offsets[-1] + 3, 2, 1, 40
    gen = generator(len(kind), causal, 61)
    q, dout = normal(gen, rows, heads, d, dtype=dtype), normal(gen, rows, heads, d, dtype=dtype)
    k, v = normal(gen, rows, kv, d, dtype=dtype), normal(gen, rows, kv, d, dtype=dtype)
    bias = normal(gen, 12, heads, dtype=dtype)
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    sequences = [s for s, n in zip(ref.ragged(offsets), lengths) if n]
    for longest, b in ((max(lengths), bias), (300, None), (1, None)):
        out, _, grads = forward_and_backward(q, k, v, dout, sequences, b, 40, causal=causal, q_offsets=at, k_offsets=at, longest_q=longest, longest_k=longest)
        for t in (out, grads.dq, grads.dk, grads.dv):
            assert not bool(t[:2].any()) and not bool(t[offsets[-1]:].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads, kv, d", [(2, 1, 64), (1, 1, 128)])
def test_parts_of_their_keys(heads, kv, d, dtype):
    rng = random.Random(d)
    batch, longest = 700, 2300
    lengths = [rng.choice([0, 1, 90, 500, 1000, 1025, 2049]) for _ in range(batch - 1)] + [longest]
    gen = generator(heads, d, 62)
    q = normal(gen, batch, 1, heads, d, dtype=dtype, scale=2.0)
    k, v = normal(gen, batch, longest, kv, d, dtype=dtype), normal(gen, batch, longest, kv, d, dtype=dtype)
    bias = normal(gen, 12, heads, dtype=dtype)
    at = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for b in (None, bias):
        out = rcd.attention(q, k, v, causal=True, k_lengths=at, bias=b, max_distance=40)
        value, bound = ref.attention(q, k, v, None, True, ref.padded(batch, lengths), b, 40)
        ref.check("out", out, value["out"], bound["out"])
