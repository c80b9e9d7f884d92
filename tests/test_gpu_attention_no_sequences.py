"""Offsets with one element: a batch of no sequences in a buffer that has rows.  All of them belong to no sequence: zeros in new results, in given
ones they are left."""
import pytest
import torch

import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, generator, normal

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def dirty(*like):
    """What the next allocations of these sizes find in their memory."""
    held = [torch.full_like(t, float("nan")) for t in like for _ in range(3)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (70, 4, 2, 64), (513, 6, 1, 33), (3000, 2, 2, 128)])
def test_both_by_offsets(size, dtype):
    rows, heads, kv, d = size
    gen = generator(rows, d, 41)
    q, dout = normal(gen, rows, heads, d, dtype=dtype), normal(gen, rows, heads, d, dtype=dtype)
    k, v = normal(gen, rows + 3, kv, d, dtype=dtype), normal(gen, rows + 3, kv, d, dtype=dtype)
    for first in (0, 1):
        at = torch.tensor([first], dtype=torch.int32, device=DEV)
        for bias in (None, normal(gen, 8, heads, dtype=dtype)):
            how = dict(q_offsets=at, k_offsets=at, bias=bias, max_distance=9)
            dirty(q, k)
            out, saved = rcd.attention(q, k, v, want_saved=True, **how)
            assert out.shape == q.shape and not bool(out.any())
            dirty(q, k, v)
            grads = rcd.attention_backward(dout, q, k, v, out, saved, **how)
            for g in grads:
                assert g is None or not bool(g.any())
            # what is given is left
            given = [torch.full_like(t, 7.0) for t in (q, k, v)]
            left = torch.full_like(q, 7.0)
            rcd.attention(q, k, v, out=left, **how)
            grads = rcd.attention_backward(dout, q, k, v, out, saved, grads=given, **how)
            assert all(bool((t == 7.0).all()) for t in [left] + given)
            assert grads.dbias is None or not bool(grads.dbias.any())


@pytest.mark.parametrize("dtype", TYPES)
def test_one_by_offsets(dtype):
    """(The other has a batch of none.)"""
    gen = generator(42)
    some, none = normal(gen, 90, 4, 40, dtype=dtype), normal(gen, 0, 50, 4, 40, dtype=dtype)
    at = torch.zeros(1, dtype=torch.int32, device=DEV)
    dirty(some)
    out, saved = rcd.attention(some, none, none, q_offsets=at, want_saved=True)
    assert not bool(out.any())
    dirty(some)
    grads = rcd.attention_backward(some, some, none, none, out, saved, q_offsets=at)
    assert not bool(grads.dq.any()) and grads.dk.shape == none.shape
    out, saved = rcd.attention(none, some, some, k_offsets=at, want_saved=True)
    assert out.shape == none.shape
    dirty(some, some)
    grads = rcd.attention_backward(none, none, some, some, out, saved, k_offsets=at)
    assert not bool(grads.dk.any()) and not bool(grads.dv.any()) and grads.dq.shape == none.shape


def test_in_a_graph():
    gen = generator(43)
    q = normal(gen, 200, 2, 64, dtype=torch.bfloat16)
    at = torch.zeros(1, dtype=torch.int32, device=DEV)
    rcd.attention(q, q, q, q_offsets=at, k_offsets=at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = rcd.attention(q, q, q, q_offsets=at, k_offsets=at)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert not bool(out.any())
