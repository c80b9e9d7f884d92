"""Attention of the feature encoder: what mixes the tokens of a sample, with the learned bias of relative positions, and its
gradients.  Argument marshalling only (csrc/encoder_marshal.cpp); the contracts stand in include/rcd.h.

q is (batch, rows, heads, d) and k, v are (batch, rows, kv_heads, d), float32 or bfloat16 device tensors whose last dimension is
contiguous (any other strides: views of one projection's result are as good as tensors of their own); heads is a multiple of
kv_heads, d at most 128.  With q_offsets, k_offsets (int32, on the device, sequence b from offset b up to offset b + 1) a tensor is
(rows, heads, d), all sequences one after the other.  The queries of a sequence stand at the end of its keys.

The rules of encoder.py hold: the current stream, a workspace unless one is given, RcdError for what cannot be served, and no
history for autograd.
"""
from __future__ import annotations

import functools
import struct
from typing import List, NamedTuple, Optional

import torch

from .encoder import _lib, _refuse, _stream


class AttentionGrads(NamedTuple):
    dq: torch.Tensor
    dk: torch.Tensor
    dv: torch.Tensor
    dbias: Optional[torch.Tensor]     # of the bias's type and shape


@functools.lru_cache(maxsize=256)
def _borders(each: int, max_distance: int) -> tuple:
    exact = each // 2
    steps = each - exact
    borders = list(range(1, exact + 1))
    r = exact
    for m in range(1, steps):
        least = exact ** (steps - m) * max_distance ** m
        while r ** steps < least:
            r += 1
        borders.append(r)
    return tuple(borders), struct.pack("=%di" % len(borders), *borders)


def _checked_borders(buckets: int, max_distance: int, causal: bool):
    each = buckets if causal else buckets // 2
    if each < 2 or (not causal and buckets % 2):
        _refuse("a bias has two buckets at least in each direction, as many behind the query as before it", 1)
    if each > 128:
        _refuse("128 buckets in a direction at most", 4)
    if not each // 2 < max_distance:
        _refuse("max_distance must be above half of a direction's buckets", 1)
    if max_distance > 1024:
        _refuse("max_distance must be 1024 at most", 4)
    return _borders(each, int(max_distance))


def position_borders(buckets: int, max_distance: int = 128, causal: bool = False) -> List[int]:
    """The distances at which the next bucket of a bias of relative positions begins.  A direction has n buckets (all of them where
    causal, else half; keys behind the query have the second half).  A distance r has bucket r below h = n // 2, from there on
    h + floor((n - h) ln(r / h) / ln(max_distance / h)), n - 1 at most; computed in whole numbers."""
    return list(_checked_borders(buckets, max_distance, causal)[0])


def _packed(bias, max_distance, causal):
    """The borders of a bias as the library takes them."""
    if bias is None:
        return None
    if not isinstance(bias, torch.Tensor) or bias.dim() != 2:
        _refuse("bias must be a contiguous tensor (buckets, heads)", 1)
    return _checked_borders(bias.shape[0], max_distance, bool(causal))[1]


def attention(q, k, v, scale=None, causal: bool = False, q_offsets=None, k_offsets=None, k_lengths=None, longest_q: int = 0,
              longest_k: int = 0, bias=None, max_distance: int = 128, out=None, want_saved: bool = False, workspace=None):
    """softmax(scale q k^T + bias) v, scale d^(-1/2) unless given.  k_lengths (int32): how many keys of each sequence there are.
    longest_q, longest_k: the longest sequence, where the caller knows it (for speed alone).  bias (buckets, heads), float32 or
    of q's type: what position_borders() makes of max_distance says which bucket a pair has.  A query that sees no key gets zeros;
    rows outside every sequence become zeros, in `out` they are left; `out` shares no elements with the rest.  want_saved: (out, saved), what attention_backward takes."""
    result, saved = _lib().attention(q, k, v, q_offsets, k_offsets, k_lengths, longest_q, longest_k, scale, causal, bias,
                                     _packed(bias, max_distance, causal), out, want_saved, workspace, _stream(q))
    return (result, saved) if want_saved else result


def attention_backward(dout, q, k, v, out, saved, scale=None, causal: bool = False, q_offsets=None, k_offsets=None, k_lengths=None,
                       longest_q: int = 0, longest_k: int = 0, bias=None, max_distance: int = 128, want_dbias: bool = True,
                       grads=None, workspace=None) -> AttentionGrads:
    """The gradients of attention's q, k, v and bias; out and saved are what it returned, the other arguments what it was given.
    grads: (dq, dk, dv) to write to, which share no elements with the rest; their rows that belong to no sequence are left (zeros in new ones)."""
    dq, dk, dv = (None, None, None) if grads is None else grads
    return AttentionGrads._make(_lib().attention_backward(
        dout, q, k, v, out, saved, q_offsets, k_offsets, k_lengths, longest_q, longest_k, scale, causal, bias,
        _packed(bias, max_distance, causal), dq, dk, dv, want_dbias, workspace, _stream(q)))
