"""Queries and keys by offsets each of its own: texts that look at other texts, keys end to end under a dense batch of queries, and strides whose
bytes pass 32 bits."""
import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, forward_and_backward, generator, normal

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def vector(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 33, 128])
def test_different_lengths(d, causal, dtype):
    """More queries than keys and fewer, none of either; queries that stand in front of the first key see nothing where causal."""
    q_at, k_at = [1, 40, 40, 45, 300, 301, 301], [0, 7, 90, 90, 350, 900, 903]
    gen = generator(d, causal, 71)
    heads, kv = 4, 2
    q, dout = normal(gen, 305, heads, d, dtype=dtype), normal(gen, 305, heads, d, dtype=dtype)
    k, v = normal(gen, 910, kv, d, dtype=dtype), normal(gen, 910, kv, d, dtype=dtype)
    sequences = [(slice(a, b), slice(c, e)) for a, b, c, e in zip(q_at[:-1], q_at[1:], k_at[:-1], k_at[1:])]
    for bias in (None, normal(gen, 16, heads, dtype=dtype)):
        for longest in ((0, 0), (255, 550), (1, 1)):
            out, _, grads = forward_and_backward(q, k, v, dout, sequences, bias, 40, causal=causal, q_offsets=vector(q_at), k_offsets=vector(k_at), longest_q=longest[0],
                                                 longest_k=longest[1])
            assert not bool(out[301:].any()) and not bool(grads.dk[903:].any()) and not bool(grads.dv[903:].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 30, 200])
def test_keys_alone_by_offsets(n, causal, dtype):
    k_at = [2, 2, 3, 320, 1500]
    gen = generator(n, causal, 72)
    heads, kv, d = 6, 2, 72
    q, dout = normal(gen, 4, n, heads, d, dtype=dtype), normal(gen, 4, n, heads, d, dtype=dtype)
    k, v = normal(gen, 1505, kv, d, dtype=dtype), normal(gen, 1505, kv, d, dtype=dtype)
    sequences = [((b, slice(None)), slice(c, e)) for b, (c, e) in enumerate(zip(k_at[:-1], k_at[1:]))]
    for bias in (None, normal(gen, 16, heads, dtype=dtype)):
        for longest in (0, 1180, 1):
            _, _, grads = forward_and_backward(q, k, v, dout, sequences, bias, 40, causal=causal, k_offsets=vector(k_at), longest_k=longest)
            assert not bool(grads.dk[:2].any()) and not bool(grads.dk[1500:].any()) and not bool(grads.dv[1500:].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 300])
def test_strides_beyond_32_bits(n, dtype):
    """Rows as far apart as they may be: the last of them begin 5 GB behind the first."""
    gen = generator(n, 73)
    heads, kv, d, m = 2, 1, 64, 300
    pitch = (2 ** 24 - 256) // torch.finfo(dtype).bits * 8
    room = torch.empty(m * pitch, dtype=dtype, device=DEV)

    def far(rows, count, first):
        return room.as_strided((1, rows, count, d), (0, pitch, d, 1), first)

    q, k, v, dk, dv = far(n, heads, 0), far(m, kv, 1024), far(m, kv, 2048), far(m, kv, 3072), far(m, kv, 4096)
    dq, dout, out = far(n, heads, 5120), far(n, heads, 6144), far(n, heads, 7168)
    for t in (q, k, v, dout):
        t.copy_(normal(gen, *t.shape, dtype=dtype))
    for causal in (False, True):
        value, bound = ref.attention(q, k, v, None, causal, ref.padded(1, [m]), None, 128, dout)
        _, saved = rcd.attention(q, k, v, causal=causal, out=out, want_saved=True)
        rcd.attention_backward(dout, q, k, v, out, saved, causal=causal, grads=(dq, dk, dv))
        for name, got in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            ref.check(name, got, value[name], bound[name])
