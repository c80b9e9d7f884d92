"""The feature encoder's operators: what turns a sample's hidden state into the feature row that similarity() and
partition_dataset() take.  Argument marshalling only, as in binding.py (the checks and the calls are in
csrc/encoder_marshal.cpp); the contracts stand in include/rcd.h.

Matrices are float32 or bfloat16 device tensors of two dimensions whose last one is contiguous (any row stride).  Where an
operator takes 8-bit operands they are float8_e4m3fn tensors with their scales beside them: uint8 or float8_e8m0fnu, one for
each 32 elements of a row.  Every call runs on the current stream; a workspace is allocated unless one is given.  What cannot
be served raises RcdError.

Autograd records none of these calls: a tensor that requires grad is refused while gradients are recorded.  Call them under
torch.no_grad(), or in the forward and backward of a torch.autograd.Function, where recording is off.
"""
from __future__ import annotations

import importlib
import os
from typing import NamedTuple, Optional

import torch

from .binding import RcdError, load_library

_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_OUT = {None: -1, torch.float32: 0, torch.bfloat16: 1}
_calls = None


class RmsNorm(NamedTuple):
    y: torch.Tensor                   # x's type, or float8_e4m3fn
    scale: Optional[torch.Tensor]     # float8_e8m0fnu, with 8-bit output
    sum: Optional[torch.Tensor]       # x + residual
    rstd: Optional[torch.Tensor]      # float32, one per row


def _lib():
    """The marshalling module, loaded behind librcd.so, which it calls."""
    global _calls
    if _calls is None:
        load_library()
        if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_encoder.so")):
            raise RcdError(-1, "_encoder.so is not built: run `python -m paper_2211_00839_amd.build`")
        _calls = importlib.import_module("._encoder", __package__)
        _calls.set_error(RcdError)
    return _calls


def _refuse(what: str, status: int):
    raise RcdError(status, what)


def _act(act: str) -> int:
    code = _ACTS.get(act)
    if code is None:
        _refuse("act must be one of %s" % ", ".join(_ACTS), 4)
    return code


def _out(dtype) -> int:
    code = _OUT.get(dtype)
    if code is None:
        _refuse("out_dtype must be float32 or bfloat16", 4)
    return code


def _stream(t) -> int:
    """The current stream of t's device (0 for what is refused further on)."""
    device = t.get_device() if isinstance(t, torch.Tensor) else -1
    return torch._C._cuda_getCurrentRawStream(device) if device >= 0 else 0


def rms_norm(x, weight=None, eps: float = 1e-6, residual=None, quantize: bool = False, want_sum: bool = False,
             want_rstd: bool = False) -> RmsNorm:
    """h = x + residual, y = h * rstd * weight with rstd = (mean h^2 + eps)^(-1/2) of each row.  quantize: y in 8 bits with
    scales.  want_sum: h too, rounded to x's type; want_rstd: what rms_norm_backward takes."""
    return RmsNorm._make(_lib().rms_norm(x, weight, eps, residual, quantize, want_sum, want_rstd, _stream(x)))


def rms_norm_backward(dy, h, rstd, weight=None, dsum=None, want_dweight: bool = True, workspace=None):
    """(dx, dweight) of rms_norm: h is its sum (x itself without a residual), rstd its rstd, dsum the gradient that reaches
    h along the residual stream.  dx is the residual's gradient too; dweight is None unless wanted."""
    return _lib().rms_norm_backward(dy, h, rstd, weight, dsum, want_dweight, workspace, _stream(dy))


def quantize_mxfp8(x):
    """(float8_e4m3fn elements, float8_e8m0fnu scales) of the rows of x."""
    return _lib().quantize_mxfp8(x, _stream(x))


def linear(a, w, bias=None, act: str = "none", residual=None, a_scale=None, w_scale=None, out_dtype=None,
           want_preact: bool = False, out=None, workspace=None):
    """act(a w^T + bias) + residual, a (M, K), w (N, K).  out may be the residual.  want_preact: (y, z), z = a w^T + bias in
    float32, what linear_backward takes."""
    y, z = _lib().linear(a, w, bias, _act(act), residual, a_scale, w_scale, _out(out_dtype), want_preact, out, workspace, _stream(a))
    return (y, z) if want_preact else y


def linear_backward(dy, a, w, preact=None, act: str = "none", want_da: bool = True, want_dw: bool = True, want_dbias: bool = True,
                    workspace=None):
    """(da, dw, dbias) of linear; preact is its z (not needed for act "none"); what is not wanted is None.  The residual's
    gradient is dy itself."""
    return _lib().linear_backward(dy, a, w, preact, _act(act), want_da, want_dw, want_dbias, workspace, _stream(dy))


def gated_linear(a, w_gate, w_up, act: str = "silu", a_scale=None, gate_scale=None, up_scale=None, out_dtype=None,
                 want_saved: bool = False, out=None, workspace=None):
    """act(a w_gate^T) * (a w_up^T), a (M, K), both weights (F, K).  want_saved: (h, saved), saved (M, F, 2) in float32 what
    gated_linear_backward takes."""
    h, saved = _lib().gated_linear(a, w_gate, w_up, _act(act), a_scale, gate_scale, up_scale, _out(out_dtype), want_saved, out,
                                   workspace, _stream(a))
    return (h, saved) if want_saved else h


def gated_linear_backward(dh, a, w_gate, w_up, saved, act: str = "silu", want_da: bool = True, want_dw: bool = True,
                          workspace=None):
    """(da, dw_gate, dw_up) of gated_linear; saved is its saved; what is not wanted is None."""
    return _lib().gated_linear_backward(dh, a, w_gate, w_up, saved, _act(act), want_da, want_dw, workspace, _stream(dh))
