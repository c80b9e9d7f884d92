"""Attention over many sequences of different lengths: workgroups go on from one to the next there, and keys are cut into parts."""
import random

import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, forward_and_backward, generator, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads", [(5, 5), (6, 3), (8, 1)])
def test_many_samples(heads, causal, dtype):
    h, kv = heads
    rng = random.Random(h)
    lengths = [rng.choice([0, 1, 2, 31, 33, 60, 130, 300]) for _ in range(60)] + [410]
    rng.shuffle(lengths)
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    rows, d = offsets[-1], 24
    gen = generator(h, causal, 11)
    q, dout = normal(gen, rows, h, d, dtype=dtype), normal(gen, rows, h, d, dtype=dtype)
    k, v = normal(gen, rows, kv, d, dtype=dtype), normal(gen, rows, kv, d, dtype=dtype)
    bias = normal(gen, 12, h, dtype=dtype)
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    for hint, b in ((410, bias), (0, None), (2000, bias)):
        forward_and_backward(q, k, v, dout, ref.ragged(offsets), b, 60, causal=causal, q_offsets=at, k_offsets=at, longest_q=hint, longest_k=hint)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(70, 6, 3, 3100, 1, 128), (23, 4, 1, 5200, 3, 64), (3, 2, 2, 9001, 2, 80), (1, 8, 1, 20000, 1, 128), (300, 2, 1, 70, 4, 64)])
def test_tokens_over_a_cache(shape, dtype):
    batch, heads, kv, longest, n, d = shape
    rng = random.Random(longest)
    lengths = [min(longest, int(longest ** rng.random()) + n) for _ in range(batch)]
    lengths[rng.randrange(batch)] = longest
    gen = generator(batch, longest, 12)
    q = normal(gen, batch, n, heads, d, dtype=dtype, scale=2.0)
    k, v = normal(gen, batch, longest, kv, d, dtype=dtype), normal(gen, batch, longest, kv, d, dtype=dtype)
    at = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    bias = normal(gen, 32, heads, dtype=dtype)
    for causal in (True, False):
        for b in (None, bias):
            out, saved = rcd.attention(q, k, v, causal=causal, k_lengths=at, bias=b, want_saved=True)
            value, bound = ref.attention(q, k, v, None, causal, ref.padded(batch, lengths), b)
            ref.check("out", out, value["out"], bound["out"])
            # what the backward call takes: the weights add up to one
            assert bool((saved[..., 0].isfinite() & saved[..., 1].isfinite()).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_in_parts(dtype):
    """Few workgroups along the keys: their queries are cut into parts whose sums are added up behind; rows behind a length get zeros."""
    gen = generator(13)
    lengths = [700, 90, 0]
    q, dout = normal(gen, 3, 900, 6, 64, dtype=dtype), normal(gen, 3, 900, 6, 64, dtype=dtype)
    k, v = normal(gen, 3, 700, 2, 64, dtype=dtype), normal(gen, 3, 700, 2, 64, dtype=dtype)
    at = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    bias = normal(gen, 16, 6, dtype=dtype)
    for causal in (False, True):
        for b in (None, bias):
            _, _, grads = forward_and_backward(q, k, v, dout, ref.padded(3, lengths), b, 40, causal=causal, k_lengths=at)
            assert not grads.dk[1, 90:].any() and not grads.dv[1, 90:].any() and not grads.dk[2].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("length", [9248, 9247, 9300])
def test_rows_that_see_fewer_tiles_than_their_sequence(length, dtype):
    """Fewer tiles of keys can make more parts of them than the whole sequence has (288 in parts of 16, 289 in parts of 17): the first queries'
    last keys count all the same."""
    gen = generator(length, 14)
    q, k, v = normal(gen, 1, 64, 1, 64, dtype=dtype), normal(gen, 1, length, 1, 64, dtype=dtype), normal(gen, 1, length, 1, 64, dtype=dtype)
    k[:, -100:] = q.mean(1, keepdim=True) * 8           # (what is seen last weighs most)
    at = torch.tensor([length], dtype=torch.int32, device=DEV)
    out = rcd.attention(q, k, v, causal=True, k_lengths=at)
    value, bound = ref.attention(q, k, v, None, True, ref.padded(1, [length]))
    ref.check("out", out, value["out"], bound["out"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("causal", [False, True])
def test_many_rows_over_parts_of_the_keys(causal, dtype):
    gen = generator(causal, 15)
    for batch, n, heads, kv, d, lengths in ((1, 4096, 1, 1, 64, [4200]), (2, 1100, 2, 1, 72, [5000, 1500]), (3, 700, 2, 2, 33, [2300, 0, 700])):
        m = max(lengths)
        q, dout = normal(gen, batch, n, heads, d, dtype=dtype), normal(gen, batch, n, heads, d, dtype=dtype)
        k, v = normal(gen, batch, m, kv, d, dtype=dtype), normal(gen, batch, m, kv, d, dtype=dtype)
        how = {} if batch == 1 else dict(k_lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))
        forward_and_backward(q, k, v, dout, ref.padded(batch, lengths), causal=causal, **how)
