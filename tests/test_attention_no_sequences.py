"""CPU tests: results of a call without sequences that are to be cleared have to be there (device pointers are made up)."""
import ctypes

import pytest

from test_attention_refusals import INVALID, OK, P, heads, lib, shape  # noqa: F401


def forward(lib, s, out, clear):  # noqa: F811
    h = [ctypes.byref(x) for x in (heads(None), heads(None), heads(None), out)]
    return lib.rcd_attention(ctypes.byref(s), *h, None, clear, P, 1 << 40, None)


def backward(lib, s, dq, dk, dv, clear):  # noqa: F811
    h = [ctypes.byref(x) for x in (heads(None), heads(None), heads(None), heads(None), heads(None), dq, dk, dv)]
    return lib.rcd_attention_backward(ctypes.byref(s), *h[:5], None, *h[5:], None, clear, P, 1 << 40, None)


def test_forward(lib):  # noqa: F811
    s = shape(batch=0, q_offsets=P, k_offsets=P)
    assert forward(lib, s, heads(None), 1) == INVALID
    assert forward(lib, s, heads(None), 0) == OK                                    # nothing is written
    assert forward(lib, shape(batch=0), heads(None), 1) == OK                       # no rows at all
    assert forward(lib, shape(batch=0, q_offsets=P, q_rows=0), heads(None), 1) == OK


@pytest.mark.parametrize("missing", range(3))
def test_backward(lib, missing):  # noqa: F811
    there = [heads(), heads(), heads()]
    there[missing] = heads(None)
    assert backward(lib, shape(batch=0, q_offsets=P, k_offsets=P), *there, 1) == INVALID
