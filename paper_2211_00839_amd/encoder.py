"""The feature encoder's operators: what turns a sample's hidden state into the feature row that similarity() and
partition_dataset() take.  Argument marshalling only, as in binding.py; the contracts stand in include/rcd.h.

Matrices are float32 or bfloat16 device tensors of two dimensions whose last one is contiguous (any row stride).  Where an
operator takes 8-bit operands they are float8_e4m3fn tensors with their scales beside them: uint8 or float8_e8m0fnu, one for
each 32 elements of a row.  Every call runs on the current stream; a workspace is allocated unless one is given.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from .binding import RcdError, _check, _dev_ptr, _stream, _workspace, load_library

_INVALID, _UNSUPPORTED = 1, 4
_BLOCK = 32
_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_CODES = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}


class RmsNorm(NamedTuple):
    y: torch.Tensor                   # x's type, or float8_e4m3fn
    scale: Optional[torch.Tensor]     # float8_e8m0fnu, with 8-bit output
    sum: Optional[torch.Tensor]       # x + residual
    rstd: Optional[torch.Tensor]      # float32, one per row


def _refuse(what: str, status: int = _INVALID):
    raise RcdError(status, what)


def _act(act: str) -> int:
    if act not in _ACTS:
        _refuse("act must be one of %s" % ", ".join(_ACTS), _UNSUPPORTED)
    return _ACTS[act]


def _matrix(name, t, rows=None, cols=None, dtype=None, like=None):
    """t, checked: a device matrix with contiguous rows, of the sizes, type and device asked for."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        _refuse("%s must be a matrix" % name)
    if not t.is_cuda:
        _refuse("%s: device tensor expected (there is no CPU path)" % name, -1)
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        _refuse("%s must be %s x %s, got %d x %d" % (name, rows, cols, t.shape[0], t.shape[1]))
    if t.shape[1] > 1 and t.shape[0] > 0 and t.stride(1) != 1:
        _refuse("the rows of %s must be contiguous" % name)
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        _refuse("the rows of %s overlap" % name)
    if t.dtype not in _CODES:
        _refuse("%s: float32, bfloat16 or float8_e4m3fn expected" % name, _UNSUPPORTED)
    if dtype is not None and t.dtype != dtype:
        _refuse("%s must be %s" % (name, dtype), _UNSUPPORTED)
    if like is not None and t.device != like.device:
        _refuse("%s is on another device" % name)
    return t


def _vector(name, t, n, dtype, like):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != n or not (t.is_contiguous() or n == 1):
        _refuse("%s must be a contiguous vector of %d" % (name, n))
    if t.dtype != dtype:
        _refuse("%s must be %s" % (name, dtype), _UNSUPPORTED)
    if t.device != like.device:
        _refuse("%s is on another device" % name)
    return t


def _scale(name, t, of):
    """The scales that belong to the 8-bit matrix `of` (None for any other type)."""
    if of.dtype != torch.float8_e4m3fn:
        if t is not None:
            _refuse("%s goes with float8_e4m3fn elements only" % name)
        return None
    blocks = -(-of.shape[1] // _BLOCK)
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.uint8, torch.float8_e8m0fnu):
        _refuse("%s (uint8 or float8_e8m0fnu) is missing" % name)
    if t.dim() != 2 or t.shape != (of.shape[0], blocks) or (blocks > 1 and t.shape[0] > 0 and t.stride(1) != 1):
        _refuse("%s must be %d x %d with contiguous rows" % (name, of.shape[0], blocks))
    if t.device != of.device:
        _refuse("%s is on another device" % name)
    return t


def _ld(t) -> int:
    """Row stride in elements (of one row it means nothing: its length)."""
    if t is None:
        return 0
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _new(rows, cols, dtype, like):
    return torch.empty((rows, cols), dtype=dtype, device=like.device)


def _here(t):
    """Calls run on the current device's stream: the tensors have to be there."""
    if t.device.index != torch.cuda.current_device():
        _refuse("tensors are on %s, the current device is another" % t.device)


def _room(workspace, nbytes, like):
    if workspace is None:
        return _workspace(nbytes, like.device)
    if not workspace.is_cuda or not workspace.is_contiguous() or workspace.dtype != torch.uint8:
        _refuse("the workspace must be a contiguous uint8 device tensor", 5)
    return workspace


def rms_norm(x, weight=None, eps: float = 1e-6, residual=None, quantize: bool = False, want_sum: bool = False,
             want_rstd: bool = False) -> RmsNorm:
    """h = x + residual, y = h * rstd * weight with rstd = (mean h^2 + eps)^(-1/2) of each row.  quantize: y in 8 bits with
    scales.  want_sum: h too, rounded to x's type; want_rstd: what rms_norm_backward takes."""
    _matrix("x", x)
    _here(x)
    rows, d = x.shape
    if residual is not None:
        _matrix("residual", residual, rows, d, x.dtype, x)
    _vector("weight", weight, d, x.dtype, x)
    y = _new(rows, d, torch.float8_e4m3fn if quantize else x.dtype, x)
    scale = _new(rows, -(-d // _BLOCK), torch.float8_e8m0fnu, x) if quantize else None
    total = _new(rows, d, x.dtype, x) if want_sum else None
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device) if want_rstd else None
    _check(load_library().rcd_rms_norm(
        _dev_ptr(x), _CODES[x.dtype], rows, d, _ld(x), _dev_ptr(residual), _ld(residual), _dev_ptr(weight), float(eps),
        _dev_ptr(total), _ld(total), _dev_ptr(y), _CODES[y.dtype], _ld(y), _dev_ptr(scale), _ld(scale), _dev_ptr(rstd), _stream()))
    return RmsNorm(y, scale, total, rstd)


def rms_norm_backward(dy, h, rstd, weight=None, dsum=None, want_dweight: bool = True, workspace=None):
    """(dx, dweight) of rms_norm: h is its sum (x itself without a residual), rstd its rstd, dsum the gradient that reaches
    h along the residual stream.  dx is the residual's gradient too; dweight is None unless wanted."""
    lib = load_library()
    _matrix("dy", dy)
    _here(dy)
    rows, d = dy.shape
    _matrix("h", h, rows, d, dy.dtype, dy)
    if rstd is None:
        _refuse("rstd is missing")
    _vector("rstd", rstd, rows, torch.float32, dy)
    _vector("weight", weight, d, dy.dtype, dy)
    if dsum is not None:
        _matrix("dsum", dsum, rows, d, dy.dtype, dy)
    dx = _new(rows, d, dy.dtype, dy)
    dweight = torch.empty(d, dtype=dy.dtype, device=dy.device) if want_dweight else None
    ws = _room(workspace, lib.rcd_rms_norm_backward_workspace_bytes(rows, d) if want_dweight else 0, dy)
    _check(lib.rcd_rms_norm_backward(
        _dev_ptr(dy), _CODES[dy.dtype], rows, d, _ld(dy), _dev_ptr(h), _ld(h), _dev_ptr(rstd), _dev_ptr(weight), _dev_ptr(dsum),
        _ld(dsum), _dev_ptr(dx), _ld(dx), _dev_ptr(dweight), _dev_ptr(ws), ws.numel(), _stream()))
    return dx, dweight


def quantize_mxfp8(x):
    """(float8_e4m3fn elements, float8_e8m0fnu scales) of the rows of x."""
    _matrix("x", x)
    _here(x)
    rows, d = x.shape
    q, scale = _new(rows, d, torch.float8_e4m3fn, x), _new(rows, -(-d // _BLOCK), torch.float8_e8m0fnu, x)
    _check(load_library().rcd_quantize_mxfp8(_dev_ptr(x), _CODES[x.dtype], rows, d, _ld(x), _dev_ptr(q), _ld(q),
                                             _dev_ptr(scale), _ld(scale), _stream()))
    return q, scale


def _out_dtype(a, out_dtype):
    if out_dtype is None:
        return torch.bfloat16 if a.dtype == torch.float8_e4m3fn else a.dtype
    if out_dtype not in (torch.float32, torch.bfloat16):
        _refuse("out_dtype must be float32 or bfloat16", _UNSUPPORTED)
    return out_dtype


def linear(a, w, bias=None, act: str = "none", residual=None, a_scale=None, w_scale=None, out_dtype=None,
           want_preact: bool = False, out=None, workspace=None):
    """act(a w^T + bias) + residual, a (M, K), w (N, K).  out may be the residual.  want_preact: (y, z), z = a w^T + bias in
    float32, what linear_backward takes."""
    lib = load_library()
    _matrix("a", a)
    _here(a)
    M, K = a.shape
    _matrix("w", w, None, K, a.dtype, a)
    N = w.shape[0]
    a_scale, w_scale = _scale("a_scale", a_scale, a), _scale("w_scale", w_scale, w)
    dt = _out_dtype(a, out_dtype) if out is None else out.dtype
    _vector("bias", bias, N, dt, a)
    if residual is not None:
        _matrix("residual", residual, M, N, dt, a)
    y = _new(M, N, dt, a) if out is None else _matrix("out", out, M, N, _out_dtype(a, out_dtype or dt), a)
    z = _new(M, N, torch.float32, a) if want_preact else None
    ws = _room(workspace, lib.rcd_linear_workspace_bytes(M, N, K, _CODES[a.dtype]), a)
    _check(lib.rcd_linear(
        _dev_ptr(a), _dev_ptr(a_scale), _ld(a), _ld(a_scale), _dev_ptr(w), _dev_ptr(w_scale), _ld(w), _ld(w_scale), _CODES[a.dtype],
        _CODES[dt], M, N, K, _dev_ptr(bias), _act(act), _dev_ptr(residual), _ld(residual), _dev_ptr(z), _ld(z), _dev_ptr(y), _ld(y),
        _dev_ptr(ws), ws.numel(), _stream()))
    return (y, z) if want_preact else y


def linear_backward(dy, a, w, preact=None, act: str = "none", want_da: bool = True, want_dw: bool = True, want_dbias: bool = True,
                    workspace=None):
    """(da, dw, dbias) of linear; preact is its z (not needed for act "none"); what is not wanted is None.  The residual's
    gradient is dy itself."""
    lib = load_library()
    _matrix("dy", dy)
    _here(dy)
    M, N = dy.shape
    _matrix("a", a, M, None, dy.dtype, dy)
    K = a.shape[1]
    _matrix("w", w, N, K, dy.dtype, dy)
    if preact is None and act != "none":
        _refuse("preact is missing")
    if preact is not None:
        _matrix("preact", preact, M, N, torch.float32, dy)
    da = _new(M, K, dy.dtype, dy) if want_da else None
    dw = _new(N, K, dy.dtype, dy) if want_dw else None
    db = torch.empty(N, dtype=dy.dtype, device=dy.device) if want_dbias else None
    ws = _room(workspace, lib.rcd_linear_backward_workspace_bytes(M, N, K, _CODES[dy.dtype]), dy)
    _check(lib.rcd_linear_backward(
        _dev_ptr(dy), _ld(dy), _dev_ptr(a), _ld(a), _dev_ptr(w), _ld(w), _CODES[dy.dtype], M, N, K, _dev_ptr(preact), _ld(preact),
        _act(act), _dev_ptr(da), _ld(da), _dev_ptr(dw), _ld(dw), _dev_ptr(db), _dev_ptr(ws), ws.numel(), _stream()))
    return da, dw, db


def gated_linear(a, w_gate, w_up, act: str = "silu", a_scale=None, gate_scale=None, up_scale=None, out_dtype=None,
                 want_saved: bool = False, out=None, workspace=None):
    """act(a w_gate^T) * (a w_up^T), a (M, K), both weights (F, K).  want_saved: (h, saved), saved (M, F, 2) in float32 what
    gated_linear_backward takes."""
    lib = load_library()
    _matrix("a", a)
    _here(a)
    M, K = a.shape
    _matrix("w_gate", w_gate, None, K, a.dtype, a)
    F = w_gate.shape[0]
    _matrix("w_up", w_up, F, K, a.dtype, a)
    a_scale = _scale("a_scale", a_scale, a)
    gate_scale, up_scale = _scale("gate_scale", gate_scale, w_gate), _scale("up_scale", up_scale, w_up)
    dt = _out_dtype(a, out_dtype) if out is None else out.dtype
    h = _new(M, F, dt, a) if out is None else _matrix("out", out, M, F, _out_dtype(a, out_dtype or dt), a)
    saved = torch.empty((M, F, 2), dtype=torch.float32, device=a.device) if want_saved else None
    ws = _room(workspace, lib.rcd_gated_linear_workspace_bytes(M, F, K, _CODES[a.dtype]), a)
    _check(lib.rcd_gated_linear(
        _dev_ptr(a), _dev_ptr(a_scale), _ld(a), _ld(a_scale), _dev_ptr(w_gate), _dev_ptr(gate_scale), _ld(w_gate), _ld(gate_scale),
        _dev_ptr(w_up), _dev_ptr(up_scale), _ld(w_up), _ld(up_scale), _CODES[a.dtype], _CODES[dt], M, F, K, _act(act),
        _dev_ptr(saved), _dev_ptr(h), _ld(h), _dev_ptr(ws), ws.numel(), _stream()))
    return (h, saved) if want_saved else h


def gated_linear_backward(dh, a, w_gate, w_up, saved, act: str = "silu", want_da: bool = True, want_dw: bool = True,
                          workspace=None):
    """(da, dw_gate, dw_up) of gated_linear; saved is its saved; what is not wanted is None."""
    lib = load_library()
    _matrix("dh", dh)
    _here(dh)
    M, F = dh.shape
    _matrix("a", a, M, None, dh.dtype, dh)
    K = a.shape[1]
    _matrix("w_gate", w_gate, F, K, dh.dtype, dh)
    _matrix("w_up", w_up, F, K, dh.dtype, dh)
    if (not isinstance(saved, torch.Tensor) or saved.shape != (M, F, 2) or saved.dtype != torch.float32
            or not saved.is_contiguous() or saved.device != dh.device):
        _refuse("saved must be what gated_linear returned")
    da = _new(M, K, dh.dtype, dh) if want_da else None
    dwg = _new(F, K, dh.dtype, dh) if want_dw else None
    dwu = _new(F, K, dh.dtype, dh) if want_dw else None
    ws = _room(workspace, lib.rcd_gated_linear_backward_workspace_bytes(M, F, K, _CODES[dh.dtype]), dh)
    _check(lib.rcd_gated_linear_backward(
        _dev_ptr(dh), _ld(dh), _dev_ptr(a), _ld(a), _dev_ptr(w_gate), _ld(w_gate), _dev_ptr(w_up), _ld(w_up), _CODES[dh.dtype],
        M, F, K, _dev_ptr(saved), _act(act), _dev_ptr(da), _ld(da), _dev_ptr(dwg), _ld(dwg), _dev_ptr(dwu), _ld(dwu),
        _dev_ptr(ws), ws.numel(), _stream()))
    return da, dwg, dwu
