"""Results that share elements with what a call reads, or with one another, are refused wherever they begin; results that lie between operands' rows
are not."""
import pytest
import torch

import paper_2211_00839_amd as rcd
from test_gpu_attention import DEV, generator, normal

pytestmark = pytest.mark.gpu


def refused(call, *a, **kw):
    with pytest.raises(rcd.RcdError):
        call(*a, **kw)


def test_out():
    gen = generator(51)
    room = normal(gen, 2, 41, 8, 64, dtype=torch.bfloat16)
    q, k, v = (t[:, :40] for t in room.split([4, 2, 2], dim=2))
    kept = room.clone()
    want = rcd.attention(q, k, v)
    for bad in (room[:, 1:, :4], room[:, 1:, 2:6], room[:, :40, 1:5], room[:, 1:, 4:], room.view(-1)[7 * 64 + 2:][:2 * 40 * 256].view(2, 40, 4, 64)):
        refused(rcd.attention, q, k, v, out=bad)
    # the operand lies inside the result's rows
    flat = torch.zeros(2 * 40 * 4 * 64 + 8, dtype=torch.bfloat16, device=DEV)
    some = flat[-136:-8].view(1, 1, 2, 64)
    refused(rcd.attention, q[:1, :40], some, some, out=flat[:40 * 4 * 64 * 2].view(1, 80, 4, 64)[:, 40:])
    assert torch.equal(room, kept)
    # another sequence's part of the buffer, heads beside the operands', the last row and on
    big = normal(gen, 4, 40, 12, 64, dtype=torch.bfloat16)
    q2, k2, v2, free = big.split([4, 2, 2, 4], dim=2)
    q2.copy_(q.repeat(2, 1, 1, 1))
    k2.copy_(k.repeat(2, 1, 1, 1))
    v2.copy_(v.repeat(2, 1, 1, 1))
    assert torch.equal(rcd.attention(q2, k2, v2, out=free), want.repeat(2, 1, 1, 1))
    assert torch.equal(rcd.attention(q2[:2], k2[:2], v2[:2], out=q2[2:]), want)


def test_beside_small_operands():
    gen = generator(52)
    q, k = normal(gen, 1, 8, 2, 64), normal(gen, 1, 9000, 2, 64)
    room = torch.zeros(4096, device=DEV)
    out = room[:1024].view(1, 8, 2, 64)
    lengths = room[1023:1024].view(torch.int32)
    refused(rcd.attention, q, k, k, k_lengths=lengths, out=out)
    rcd.attention(q, k, k, k_lengths=room[1024:1025].view(torch.int32), out=out)
    bias = room[1000:1016].view(8, 2)
    refused(rcd.attention, q, k, k, bias=bias, max_distance=9, out=out)
    # the workspace's bytes that are used
    at = torch.tensor([9000], dtype=torch.int32, device=DEV)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    want = rcd.attention(q, k, k, k_lengths=at, workspace=ws)
    refused(rcd.attention, q, k, k, k_lengths=at, workspace=ws, out=ws[64:64 + 4096].view(torch.float32).view(1, 8, 2, 64))
    behind = ws[-4096:].view(torch.float32).view(1, 8, 2, 64)
    assert torch.equal(rcd.attention(q, k, k, k_lengths=at, workspace=ws, out=behind), want)


def test_gradients():
    gen = generator(53)
    at = torch.tensor([0, 30, 60], dtype=torch.int32, device=DEV)
    how = dict(q_offsets=at, k_offsets=at)
    qkv, dqkv = normal(gen, 60, 8, 40), torch.zeros(60, 8, 40, device=DEV)
    q, k, v = qkv.split([4, 2, 2], dim=1)
    dout = normal(gen, 60, 4, 40)
    out, saved = rcd.attention(q, k, v, want_saved=True, **how)
    want = rcd.attention_backward(dout, q, k, v, out, saved, **how)

    def call(dq, dk, dv):
        return rcd.attention_backward(dout, q, k, v, out, saved, grads=(dq, dk, dv), **how)

    dq, dk, dv = dqkv.split([4, 2, 2], dim=1)
    assert all(torch.equal(a, b) for a, b in zip(call(dq, dk, dv)[:3], want[:3]))
    refused(call, dq, dqkv[:, 3:5], dv)
    refused(call, dq, dk, dqkv[:, 5:7])
    refused(call, dqkv[:, 2:6], dk, dv)
    refused(call, dq, dk, qkv[:, 6:])
    more = torch.zeros(61, 4, 40, device=DEV)
    more[1:] = dout
    refused(rcd.attention_backward, more[1:], q, k, v, out, saved, grads=(more[:60], dk, dv), **how)
    line = torch.zeros(60 * 4 * 40 + 480, device=DEV)
    line[480:] = saved.reshape(-1).repeat(20)
    refused(rcd.attention_backward, dout, q, k, v, out, line[480:960].view(60, 4, 2), grads=(line[:9600].view(60, 4, 40), dk, dv), **how)
    torch.cuda.synchronize()
