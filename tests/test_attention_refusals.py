"""CPU tests: what attention's entry points refuse, before anything is launched (device pointers are made up: a call that touched one would
not come back with the status asked for), and the borders of the position bias."""
import ctypes
import math
import os

import pytest
import torch

import attention_reference as ref
import paper_2211_00839_amd as rcd

P = 1 << 20      # any aligned address
F32, BF16, MX = 0, 1, 2
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 4, 5


class Heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("batch", ctypes.c_int64), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class Shape(ctypes.Structure):
    _fields_ = ([("dt", ctypes.c_int)] + [(n, ctypes.c_int64) for n in ("batch", "heads", "kv_heads", "d", "q_rows", "k_rows")] +
                [(n, ctypes.c_void_p) for n in ("q_offsets", "k_offsets", "k_lengths")] + [("longest_q", ctypes.c_int64), ("longest_k", ctypes.c_int64)] +
                [("causal", ctypes.c_int), ("scale", ctypes.c_float), ("bias", ctypes.c_void_p), ("bias_dt", ctypes.c_int), ("buckets", ctypes.c_int64),
                 ("borders", ctypes.c_void_p)])


@pytest.fixture(scope="module")
def lib():
    from paper_2211_00839_amd import binding
    if not os.path.exists(binding.lib_path()):
        from paper_2211_00839_amd import build
        build.build()
    return binding.load_library()


KEEP = []


def shape(**change):
    borders = change.pop("borders", None)
    s = Shape(dt=BF16, batch=2, heads=4, kv_heads=2, d=64, q_rows=8, k_rows=8, scale=0.125)
    for name, value in change.items():
        setattr(s, name, value)
    if borders is not None:
        b = (ctypes.c_int32 * max(len(borders), 1))(*borders)
        KEEP.append(b)
        s.borders = ctypes.cast(b, ctypes.c_void_p)
    return s


def heads(p=P, batch=2048, row=256, head=64):
    return Heads(p, batch, row, head)


def forward(lib, s=None, q=None, k=None, v=None, out=None, ws=P, nbytes=1 << 40, null=False):
    h = [ctypes.byref(x if x is not None else heads()) for x in (q, k, v, out)]
    return lib.rcd_attention(None if null else ctypes.byref(s or shape()), *h, None, 0, ws, nbytes, None)


def backward(lib, s=None, dbias=None, saved=P, ws=P, nbytes=1 << 40, change=None):
    h = [heads() for _ in range(8)]
    if change:
        h[change[0]] = change[1]
    h = [ctypes.byref(x) for x in h]
    return lib.rcd_attention_backward(ctypes.byref(s or shape()), *h[:5], saved, *h[5:], dbias, 0, ws, nbytes, None)


BAD_SHAPES = [(dict(dt=MX), UNSUPPORTED), (dict(dt=7), UNSUPPORTED), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID),
              (dict(d=0), INVALID), (dict(d=129), UNSUPPORTED), (dict(batch=-1), INVALID), (dict(q_rows=-1), INVALID), (dict(k_rows=-1), INVALID),
              (dict(longest_q=-1), INVALID), (dict(longest_k=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
              (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=1e-40), INVALID), (dict(scale=3e38), INVALID),
              (dict(q_rows=2 ** 30), UNSUPPORTED), (dict(k_rows=2 ** 30), UNSUPPORTED), (dict(batch=2 ** 24), UNSUPPORTED), (dict(heads=2 ** 16, kv_heads=1), UNSUPPORTED),
              (dict(k_offsets=P, k_lengths=P), INVALID),
              (dict(bias=P, bias_dt=F32, buckets=8), INVALID), (dict(bias=P, bias_dt=MX, buckets=8, borders=[1, 2, 3]), UNSUPPORTED),
              (dict(bias=P, buckets=7, borders=[1, 2, 3]), INVALID), (dict(bias=P, buckets=2, borders=[1]), INVALID), (dict(bias=P, buckets=1, causal=1, borders=[1]), INVALID),
              (dict(bias=P, buckets=8, borders=[0, 2, 3]), INVALID), (dict(bias=P, buckets=8, borders=[1, 3, 2]), INVALID),
              (dict(bias=P, buckets=8, borders=[1, 2, 1025]), UNSUPPORTED), (dict(bias=P, buckets=258, borders=list(range(1, 129))), UNSUPPORTED),
              (dict(bias=P, buckets=129, causal=1, borders=list(range(1, 129))), UNSUPPORTED)]


@pytest.mark.parametrize("change, status", BAD_SHAPES)
def test_shapes(lib, change, status):
    change = dict(change)
    if "bias" in change:
        change.setdefault("bias_dt", BF16)
    s = shape(**change)
    assert forward(lib, s) == status
    assert backward(lib, s) == status
    assert lib.rcd_attention_workspace_bytes(ctypes.byref(s)) == 0
    assert lib.rcd_attention_backward_workspace_bytes(ctypes.byref(s)) == 0


def test_forward(lib):
    assert forward(lib, null=True) == INVALID
    assert forward(lib, shape(batch=0)) == OK
    assert forward(lib, shape(q_rows=0), q=heads(None), out=heads(None)) == OK
    for i in range(4):
        for bad, status in ((heads(None), INVALID), (heads(row=-1), INVALID), (heads(batch=-1), INVALID), (heads(head=-1), INVALID), (heads(row=2 ** 23), UNSUPPORTED)):
            h = [None] * 4
            h[i] = bad
            assert forward(lib, None, *h) == status
    # a long cache: its parts take a workspace
    long = shape(batch=1, q_rows=1, k_rows=100000, heads=16, kv_heads=2, d=128)
    need = lib.rcd_attention_workspace_bytes(ctypes.byref(long))
    assert need > 0 and need % 256 == 0
    assert forward(lib, long, ws=None) == WORKSPACE
    assert forward(lib, long, ws=P + 8) == WORKSPACE
    assert forward(lib, long, nbytes=need - 1) == WORKSPACE
    assert lib.rcd_attention_workspace_bytes(ctypes.byref(shape())) == 0


def test_backward(lib):
    assert backward(lib, saved=None) == INVALID
    assert backward(lib, dbias=P) == INVALID                        # no bias that it would be the gradient of
    for i in range(8):
        assert backward(lib, change=(i, heads(None))) == INVALID
        assert backward(lib, change=(i, heads(row=-1))) == INVALID
    need = lib.rcd_attention_backward_workspace_bytes(ctypes.byref(shape()))
    assert need > 0 and need % 256 == 0
    assert backward(lib, ws=None) == WORKSPACE
    assert backward(lib, ws=P + 8) == WORKSPACE
    assert backward(lib, nbytes=need - 1) == WORKSPACE


def test_borders():
    """Against the definition by whole powers, and the published form with its logarithm wherever that is not next to a border."""
    for causal in (False, True):
        for buckets in (4, 6, 8, 18, 32, 64, 128):
            n = buckets if causal else buckets // 2
            for distance in (n // 2 + 1, n // 2 + 3, 50, 128, 300, 1024):
                if distance <= n // 2:
                    continue
                borders = rcd.position_borders(buckets, distance, causal)
                assert len(borders) == n - 1 and borders == sorted(borders) and borders[0] == 1 and borders[-1] <= max(distance, n // 2)
                table = ref.bucket_table(buckets, distance, causal)
                for r in range(distance + 1):
                    assert sum(b <= r for b in borders) == table[r], (buckets, distance, r)
                    if r > n // 2:
                        x = n // 2 + (n - n // 2) * math.log(r / (n // 2)) / math.log(distance / (n // 2))
                        if abs(x - round(x)) > 1e-9:
                            assert table[r] == min(int(x), n - 1)


def refused(status, call, *a, **k):
    with pytest.raises(rcd.RcdError) as e:
        call(*a, **k)
    assert e.value.status == status, (e.value, e.value.status)


def test_python_calls():
    for buckets, distance, causal, status in ((3, 128, False, INVALID), (2, 128, False, INVALID), (1, 128, True, INVALID), (8, 2, False, INVALID), (8, 1025, False, UNSUPPORTED),
                                              (260, 1000, False, UNSUPPORTED), (129, 1000, True, UNSUPPORTED)):
        refused(status, rcd.position_borders, buckets, distance, causal)
    q = torch.zeros(2, 4, 2, 8)
    refused(-1, rcd.attention, q, q, q)                              # not on the device
    refused(INVALID, rcd.attention, None, q, q)
    refused(INVALID, rcd.attention, q[0], q, q)                      # three dimensions go with offsets
    refused(INVALID, rcd.attention, q, q, q, bias=torch.zeros(8))
    refused(INVALID, rcd.attention, q, q, q, bias=torch.zeros(7, 2))
    refused(UNSUPPORTED, rcd.attention, q.clone().requires_grad_(), q, q)


def test_the_definition_against_differences():
    """The gradients that the GPU tests compare with, against differences of the definition itself."""
    gen = torch.Generator().manual_seed(3)
    n, m, d = 5, 7, 6
    q, k, v, dout = (torch.randn(r, d, generator=gen, dtype=torch.float64) for r in (n, m, m, n))
    bias = torch.randn(8, generator=gen, dtype=torch.float64)
    for causal in (False, True):
        offset = torch.arange(m)[None, :] - (torch.arange(n) + (m - n))[:, None]
        bucket = ref.buckets_of(offset, 8, 5, causal)
        value, _ = ref.one_head(q, k, v, 0.4, causal, bias, bucket, dout)
        for name, t in (("dq", q), ("dk", k), ("dv", v), ("dbias", bias)):
            for at in [(0,) * t.dim(), tuple(s - 1 for s in t.shape), tuple(s // 2 for s in t.shape)]:
                sums = []
                for step in (1e-5, -1e-5):
                    kept = t[at].item()
                    t[at] = kept + step
                    sums.append((ref.one_head(q, k, v, 0.4, causal, bias, bucket)[0]["out"] * dout).sum().item())
                    t[at] = kept
                assert abs((sums[0] - sums[1]) / 2e-5 - value[name][at].item()) < 1e-8, (name, at)
