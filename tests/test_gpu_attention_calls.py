"""Calls of attention that its documentation allows beside the plain ones: any strides, results in given tensors, biases that mask, streams and
captured graphs, and a run of the encoder's operators together."""
import math

import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, forward_and_backward, generator, normal

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


def same(a, b):
    return a.shape == b.shape and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 150])
def test_strides(n, dtype):
    """Odd addresses and strides, heads before rows, heads that share memory: the same values give the same results as contiguous tensors' within
    what the order of loads may not change, none at all."""
    gen = generator(n, 21)
    heads, kv, d = 4, 2, 40
    room = normal(gen, 2 * (n + 3) * (heads + 2 * kv) * (d + 3) + 1, dtype=dtype)
    packed = room[1:].view(2, n + 3, heads + 2 * kv, d + 3)[:, 2:2 + n, :, 1:1 + d]
    q, k, v = packed.split([heads, kv, kv], dim=2)
    dout = normal(gen, 2, heads, n, d, dtype=dtype).transpose(1, 2)
    out, saved, grads = forward_and_backward(q, k, v, dout, ref.padded(2, [n, n]), causal=True)
    c = [t.contiguous() for t in (q, k, v, dout)]
    out2, saved2 = rcd.attention(c[0], c[1], c[2], causal=True, want_saved=True)
    grads2 = rcd.attention_backward(c[3], c[0], c[1], c[2], out2, saved2, causal=True)
    assert same(out, out2) and same(saved, saved2)
    assert all(same(a, b) for a, b in zip(grads[:3], grads2[:3]))
    # one head of k and v, read by all
    one, other = k[:, :, :1].expand(-1, -1, heads, -1), v[:, :, :1].expand(-1, -1, heads, -1)
    a, b = rcd.attention(q, one, other), rcd.attention(q, one.contiguous(), other.contiguous())
    assert same(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 33])
def test_results_in_given_tensors(d, dtype):
    """Results go where they are told to and nowhere else; rows that belong to no sequence are left."""
    gen = generator(d, 22)
    offsets, rows, heads, kv = [2, 90, 91, 230], 240, 4, 2
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    qkv, dout = normal(gen, rows, heads + 2 * kv, d, dtype=dtype), normal(gen, rows, heads, d, dtype=dtype)
    q, k, v = qkv.split([heads, kv, kv], dim=1)
    how = dict(q_offsets=at, k_offsets=at, causal=True)
    want, saved = rcd.attention(q, k, v, want_saved=True, **how)
    grads = rcd.attention_backward(dout, q, k, v, want, saved, **how)
    room = torch.full((rows, heads + 1, d + 5), 7.0, dtype=dtype, device=DEV)
    out = room[:, :heads, 3:3 + d]
    assert rcd.attention(q, k, v, out=out, **how).data_ptr() == out.data_ptr()
    inside = slice(offsets[0], offsets[-1])
    assert same(out[inside], want[inside]) and not want[:2].any() and not want[230:].any()
    expected = torch.full_like(room, 7.0)
    expected[inside, :heads, 3:3 + d] = want[inside]
    assert same(room, expected)
    droom = torch.full((rows, heads + 2 * kv, d), 7.0, dtype=dtype, device=DEV)
    into = droom.split([heads, kv, kv], dim=1)
    rcd.attention_backward(dout, q, k, v, want, saved, grads=into, **how)
    for a, b in zip(into, grads[:3]):
        assert same(a[inside], b[inside]) and not b[:2].any() and not b[230:].any()
        assert bool((a[:2] == 7.0).all()) and bool((a[230:] == 7.0).all())
    # dense: keys behind their lengths
    k, v = normal(gen, 2, 50, kv, d, dtype=dtype), normal(gen, 2, 50, kv, d, dtype=dtype)
    q, dout = normal(gen, 2, 20, heads, d, dtype=dtype), normal(gen, 2, 20, heads, d, dtype=dtype)
    lengths = torch.tensor([50, 13], dtype=torch.int32, device=DEV)
    out, saved = rcd.attention(q, k, v, k_lengths=lengths, want_saved=True)
    grads = rcd.attention_backward(dout, q, k, v, out, saved, k_lengths=lengths)
    into = [torch.full_like(t, 7.0) for t in (q, k, v)]
    rcd.attention_backward(dout, q, k, v, out, saved, k_lengths=lengths, grads=into)
    assert same(into[0], grads.dq)
    for a, b in zip(into[1:], grads[1:3]):
        assert same(a[0], b[0]) and same(a[1, :13], b[1, :13]) and bool((a[1, 13:] == 7.0).all()) and not b[1, 13:].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, m", [(1, 3000), (40, 40), (300, 300)])
def test_bias_that_masks(n, m, dtype):
    gen = generator(n, 23)
    heads, d, half = 2, 64, torch.finfo(dtype).eps / 2
    q, dout = normal(gen, 1, n, heads, d, dtype=dtype), normal(gen, 1, n, heads, d, dtype=dtype)
    k, v = normal(gen, 1, m, heads, d, dtype=dtype), normal(gen, 1, m, heads, d, dtype=dtype)
    # minus infinity for a whole side and for single buckets
    for buckets in ([7], [3], [0, 5], [3, 7], list(range(4, 8))):
        bias = normal(gen, 8, heads, dtype=dtype)
        bias[buckets, 0] = -math.inf
        forward_and_backward(q, k, v, dout, ref.padded(1, [m]), bias, 20)
    # nothing is left for any query: zeros, and no gradient
    bias = torch.full((8, heads), -math.inf, dtype=dtype, device=DEV)
    out, saved = rcd.attention(q, k, v, bias=bias, max_distance=20, want_saved=True)
    grads = rcd.attention_backward(dout, q, k, v, out, saved, bias=bias, max_distance=20)
    assert not out.any() and not any(bool(g.any()) for g in grads)
    # the type's lowest value everywhere: it swallows the scores, every key weighs the same
    for lowest in (torch.finfo(dtype).min, torch.finfo(torch.bfloat16).min):
        bias = torch.full((8, heads), lowest, dtype=dtype, device=DEV)
        out, saved = rcd.attention(q, k, v, bias=bias, max_distance=20, want_saved=True)
        mean, size = v.double().mean(1, keepdim=True).expand(1, n, heads, d), v.double().abs().mean(1, keepdim=True)
        ref.check("out", out, mean.contiguous(), ((half if dtype == torch.bfloat16 else 0) + 2 * (m + 32) * ref.U) * size + half * mean.abs())
        dv = rcd.attention_backward(dout, q, k, v, out, saved, bias=bias, max_distance=20).dv
        want = (dout.double().sum(1, keepdim=True) / m).expand(1, m, heads, d).contiguous()
        size = dout.double().abs().sum(1, keepdim=True) / m
        ref.check("dv", dv, want, ((half if dtype == torch.bfloat16 else 0) + 2 * (m + n + 32) * ref.U) * size + half * want.abs())
        # and where some are ordinary, those alone count
        bias[:4] = 0.0
        out = rcd.attention(q, k, v, bias=bias, max_distance=20)
        b = bias.clone()
        b[4:] = -math.inf
        assert same(out, rcd.attention(q, k, v, bias=b, max_distance=20))


def test_offsets_and_lengths_out_of_range():
    """They are held inside the tensors."""
    gen = generator(24)
    q = normal(gen, 70, 2, 64, dtype=torch.bfloat16)
    want = rcd.attention(q[None], q[None], q[None])[0]
    at = torch.tensor([-5, 2 ** 30], dtype=torch.int32, device=DEV)
    assert same(rcd.attention(q, q, q, q_offsets=at, k_offsets=at), want)
    at = torch.tensor([0, 40, 20, 500], dtype=torch.int32, device=DEV)
    rcd.attention(q, q, q, q_offsets=at, k_offsets=at)
    out, saved = rcd.attention(q, q, q, q_offsets=at, k_offsets=at, want_saved=True)
    rcd.attention_backward(q, q, q, q, out, saved, q_offsets=at, k_offsets=at)
    lengths = torch.tensor([2 ** 30], dtype=torch.int32, device=DEV)
    assert same(rcd.attention(q[None], q[None], q[None], k_lengths=lengths)[0], want)
    lengths.fill_(-3)
    assert not rcd.attention(q[None], q[None], q[None], k_lengths=lengths).any()
    torch.cuda.synchronize()


def test_nothing_at_all():
    gen = generator(25)
    for n, m, batch in ((0, 5, 2), (5, 0, 2), (0, 0, 2), (5, 5, 0)):
        q, k = normal(gen, batch, n, 2, 16), normal(gen, batch, m, 2, 16)
        bias = normal(gen, 8, 2)
        out, saved = rcd.attention(q, k, k, bias=bias, max_distance=9, want_saved=True)
        grads = rcd.attention_backward(q, q, k, k, out, saved, bias=bias, max_distance=9)
        assert out.shape == q.shape and grads.dk.shape == k.shape and not out.any() and not any(bool(g.any()) for g in grads)
    at = torch.zeros(4, dtype=torch.int32, device=DEV)
    q = normal(gen, 6, 2, 16)
    out, saved = rcd.attention(q, q, q, q_offsets=at, k_offsets=at, want_saved=True)
    grads = rcd.attention_backward(q, q, q, q, out, saved, q_offsets=at, k_offsets=at)
    assert not out.any() and not any(bool(g.any()) for g in grads[:3])


def test_refusals():
    gen = generator(26)
    q = normal(gen, 2, 8, 4, 64, dtype=torch.bfloat16)
    k = normal(gen, 2, 9, 2, 64, dtype=torch.bfloat16)
    at = torch.tensor([0, 8], dtype=torch.int32, device=DEV)

    def refused(call, *a, **kw):
        with pytest.raises(rcd.RcdError):
            call(*a, **kw)

    refused(rcd.attention, q, k.float(), k)
    refused(rcd.attention, q.half(), k.half(), k.half())
    refused(rcd.attention, q, k, k[:, :8])
    refused(rcd.attention, q, k[..., :32], k[..., :32])
    refused(rcd.attention, q[:, :, :3], k, k)
    refused(rcd.attention, q, k[:1], k[:1])
    refused(rcd.attention, q.transpose(2, 3), k, k)
    refused(rcd.attention, q, k, k, q_offsets=at)
    refused(rcd.attention, q[0], k, k, q_offsets=at.long())
    refused(rcd.attention, q[0], k, k, q_offsets=at.cpu())
    refused(rcd.attention, q[0], k, k, q_offsets=torch.zeros(7, dtype=torch.int32, device=DEV))
    refused(rcd.attention, q, k, k, k_lengths=at[:1])
    refused(rcd.attention, q, k, k, scale=0.0)
    refused(rcd.attention, q, k, k, scale=float("nan"))
    refused(rcd.attention, q, k, k, longest_q=-1)
    refused(rcd.attention, q, k, k, bias=torch.zeros(8, 3, dtype=torch.bfloat16, device=DEV))
    refused(rcd.attention, q, k, k, bias=torch.zeros(8, 4, dtype=torch.half, device=DEV))
    refused(rcd.attention, q, k, k, bias=torch.zeros(8, 4))
    refused(rcd.attention, q, k, k, bias=torch.zeros(8, 8, device=DEV)[:, ::2])
    refused(rcd.attention, q, k, k, out=q[:1].expand(2, -1, -1, -1))
    refused(rcd.attention, q, k, k, out=torch.empty_like(q, dtype=torch.float32))
    refused(rcd.attention, q, k, k, out=torch.empty_like(q)[:, :4])
    refused(rcd.attention, torch.zeros(1, 2, 1, 136, device=DEV), torch.zeros(1, 2, 1, 136, device=DEV), torch.zeros(1, 2, 1, 136, device=DEV))
    out, saved = rcd.attention(q, k, k, want_saved=True)
    refused(rcd.attention_backward, q, q, k, k, out, saved[:, :4])
    refused(rcd.attention_backward, q, q, k, k, out, None)
    refused(rcd.attention_backward, q[:, :4], q, k, k, out, saved)
    refused(rcd.attention_backward, q, q, k, k, out, saved, grads=(torch.empty_like(q), None, torch.empty_like(k)))
    refused(rcd.attention_backward, q, q, k, k, out, saved, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    refused(rcd.attention, q, q, q, out=q)
    refused(rcd.attention_backward, q, q, k, k, out, saved, grads=(out, torch.empty_like(k), torch.empty_like(k)))
    both = torch.empty_like(k)
    refused(rcd.attention_backward, q, q, k, k, out, saved, grads=(torch.empty_like(q), both, both))
    refused(rcd.attention, q.clone().requires_grad_(), k, k)
    with torch.no_grad():
        rcd.attention(q.clone().requires_grad_(), k, k)
    torch.cuda.synchronize()


def test_graphs_and_streams():
    """Captured once and replayed with new inputs in the same places, eager work between the replays; two graphs that share a workspace; another
    stream.  Everything comes out as the eager calls' bits."""
    gen = generator(27)
    offsets = [0, 100, 130, 400]
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    q, dout = normal(gen, 400, 4, 64, dtype=torch.bfloat16), normal(gen, 400, 4, 64, dtype=torch.bfloat16)
    k, v = normal(gen, 400, 2, 64, dtype=torch.bfloat16), normal(gen, 400, 2, 64, dtype=torch.bfloat16)
    bias = normal(gen, 16, 4, dtype=torch.bfloat16)
    cache_q, cache = normal(gen, 1, 1, 4, 64, dtype=torch.bfloat16), normal(gen, 1, 9000, 2, 64, dtype=torch.bfloat16)
    length = torch.tensor([9000], dtype=torch.int32, device=DEV)
    workspace = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)

    def train():
        out, saved = rcd.attention(q, k, v, q_offsets=at, k_offsets=at, longest_q=270, bias=bias, want_saved=True, workspace=workspace)
        return (out, saved) + tuple(rcd.attention_backward(dout, q, k, v, out, saved, q_offsets=at, k_offsets=at, longest_q=270, bias=bias, workspace=workspace))

    def serve():
        return (rcd.attention(cache_q, cache, cache, causal=True, k_lengths=length, workspace=workspace),)

    def agree(one, other, rows):
        # (what is saved of rows that belong to no sequence is not written)
        return all(same(a[:rows], b[:rows]) if a.shape == (400, 4, 2) else same(a, b) for a, b in zip(one, other))

    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for call in (train, serve):
            call()
            call()
    torch.cuda.current_stream().wait_stream(side)
    for call in (train, serve):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            made = call()
        graphs.append((g, made, call))
    for replay in range(4):
        q.copy_(normal(gen, 400, 4, 64))
        cache_q.copy_(normal(gen, 1, 1, 4, 64))
        at.copy_(torch.tensor([0, 100 + replay, 130, 400 - replay], dtype=torch.int32))
        length.fill_(9000 - 2500 * replay)
        for g, made, call in graphs:
            g.replay()
        for g, made, call in graphs:
            eager = [t.clone() for t in call()]
            assert agree(made, eager, 400 - replay), (replay, call.__name__)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = train()
    torch.cuda.current_stream().wait_stream(side)
    here = train()
    torch.cuda.synchronize()
    assert agree(there, here, 397)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_layer(dtype):
    """Norm, projection, attention with its bias over samples end to end, projection back with the residual, and all their gradients: attention's part
    against the definition on what the operators around it made, the projection's gradient against the gradients that attention put side by side."""
    gen = generator(28)
    offsets, width, heads, kv, d = [0, 60, 61, 190], 128, 4, 2, 32
    rows, inner = offsets[-1], (heads + 2 * kv) * d
    at = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    x = normal(gen, rows, width, dtype=dtype)
    w_in, w_out = normal(gen, inner, width, dtype=dtype, scale=width ** -0.5), normal(gen, width, heads * d, dtype=dtype, scale=(heads * d) ** -0.5)
    bias = normal(gen, 32, heads, dtype=dtype)
    how = dict(q_offsets=at, k_offsets=at, longest_q=129, longest_k=129, bias=bias)
    n = rcd.rms_norm(x, want_rstd=True)
    qkv = rcd.linear(n.y, w_in).view(rows, heads + 2 * kv, d)
    q, k, v = qkv.split([heads, kv, kv], dim=1)
    mixed, saved = rcd.attention(q, k, v, want_saved=True, **how)
    y = rcd.linear(mixed.view(rows, heads * d), w_out, residual=x)
    dy = normal(gen, rows, width, dtype=dtype)
    dmixed, dw_out, _ = rcd.linear_backward(dy, mixed.view(rows, heads * d), w_out, want_dbias=False)
    dmixed = dmixed.view(rows, heads, d)
    dqkv = torch.empty_like(qkv)
    grads = rcd.attention_backward(dmixed, q, k, v, mixed, saved, grads=dqkv.split([heads, kv, kv], dim=1), **how)
    dn, dw_in, _ = rcd.linear_backward(dqkv.view(rows, inner), n.y, w_in, want_dbias=False)
    dx, _ = rcd.rms_norm_backward(dn, x, n.rstd, dsum=dy, want_dweight=False)
    value, bound = ref.attention(q, k, v, None, False, ref.ragged(offsets), bias, 128, dmixed)
    ref.check("out", mixed, value["out"], bound["out"])
    for name in ("dq", "dk", "dv", "dbias"):
        ref.check(name, getattr(grads, name), value[name], bound[name])
    half = torch.finfo(dtype).eps / 2
    g, w = dqkv.view(rows, inner).double(), w_in.double()
    ref.check("dn", dn, g @ w, (inner + 32) * 2 ** -22 * (g.abs() @ w.abs()) + half * (g @ w).abs() + 1e-30)
    a = n.y.double()
    ref.check("dw", dw_in, g.t() @ a, (rows + 32) * 2 ** -22 * (g.abs().t() @ a.abs()) + half * (g.t() @ a).abs() + 1e-30)
    assert y.isfinite().all() and dx.isfinite().all() and dw_out.isfinite().all()
