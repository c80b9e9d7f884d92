"""The feature encoder's operators: what turns a sample's hidden state into the feature row that similarity() and
partition_dataset() take.  Argument marshalling only, as in binding.py; the contracts stand in include/rcd.h.

Matrices are float32 or bfloat16 device tensors of two dimensions whose last one is contiguous (any row stride).  Where an
operator takes 8-bit operands they are float8_e4m3fn tensors with their scales beside them: uint8 or float8_e8m0fnu, one for
each 32 elements of a row.  Every call runs on the current stream; a workspace is allocated unless one is given.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from .binding import RcdError, _check, _workspace, load_library

_INVALID, _UNSUPPORTED = 1, 4
_BLOCK = 32
_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_F32, _BF16, _E4M3, _E8M0 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
_CODES = {_F32: 0, _BF16: 1, _E4M3: 2}


class RmsNorm(NamedTuple):
    y: torch.Tensor                   # x's type, or float8_e4m3fn
    scale: Optional[torch.Tensor]     # float8_e8m0fnu, with 8-bit output
    sum: Optional[torch.Tensor]       # x + residual
    rstd: Optional[torch.Tensor]      # float32, one per row


def _refuse(what: str, status: int = _INVALID):
    raise RcdError(status, what)


def _act(act: str) -> int:
    code = _ACTS.get(act)
    if code is None:
        _refuse("act must be one of %s" % ", ".join(_ACTS), _UNSUPPORTED)
    return code


# The checks are written for the good case: a call of a few microseconds is what a single sample takes, and attribute by
# attribute they would cost as much as its kernel.  _why() looks again, for the message.

def _first(name, t):
    """(rows, columns, leading dimension, type, device index) of a call's first matrix, which the others have to match."""
    if isinstance(t, torch.Tensor) and t.dim() == 2 and t.dtype in _CODES and t.is_cuda:
        rows, cols = t.shape
        ld, one = t.stride()
        if (one == 1 or cols <= 1 or rows == 0) and (ld >= cols or rows <= 1):
            device = t.get_device()
            if device != torch.cuda.current_device():
                _refuse("%s is on another device than the current one" % name)
            return rows, cols, ld if rows > 1 else max(cols, 1), t.dtype, device
    _why(name, t, None, None, None, None)


def _other(name, t, rows, cols, dtype, device):
    """The leading dimension of a matrix that has to be rows x cols (rows None: any)."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.dim() == 2:
        n, d = t.shape
        if (n == rows or rows is None) and d == cols:
            ld, one = t.stride()
            if (one == 1 or cols <= 1 or n == 0) and (ld >= cols or n <= 1):
                return ld if n > 1 else max(cols, 1)
    _why(name, t, rows, cols, dtype, device)


def _why(name, t, rows, cols, dtype, device):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        _refuse("%s must be a matrix" % name)
    if not t.is_cuda:
        _refuse("%s: device tensor expected (there is no CPU path)" % name, -1)
    if t.dtype not in _CODES:
        _refuse("%s: float32, bfloat16 or float8_e4m3fn expected" % name, _UNSUPPORTED)
    if dtype is not None and t.dtype != dtype:
        _refuse("%s must be %s" % (name, dtype), _UNSUPPORTED)
    if device is not None and t.get_device() != device:
        _refuse("%s is on another device" % name)
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        _refuse("%s must be %s x %s, got %d x %d" % (name, "any" if rows is None else rows, cols, t.shape[0], t.shape[1]))
    if t.shape[1] > 1 and t.stride(1) != 1:
        _refuse("the rows of %s must be contiguous" % name)
    _refuse("the rows of %s overlap" % name)


def _vector(name, t, n, dtype, device):
    """The address of a contiguous vector, None for None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != n or not (n <= 1 or t.stride(0) == 1):
        _refuse("%s must be a contiguous vector of %d" % (name, n))
    if t.dtype is not dtype:
        _refuse("%s must be %s" % (name, dtype), _UNSUPPORTED)
    if t.get_device() != device:
        _refuse("%s is on another device" % name)
    return t.data_ptr()


def _scale(name, t, dtype, rows, cols, device):
    """(address, leading dimension) of the scales that belong to an 8-bit matrix; (None, 0) for any other type."""
    if dtype is not _E4M3:
        if t is not None:
            _refuse("%s goes with float8_e4m3fn elements only" % name)
        return None, 0
    blocks = -(-cols // _BLOCK)
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.uint8, _E8M0):
        _refuse("%s (uint8 or float8_e8m0fnu) is missing" % name)
    if t.dim() != 2 or t.shape != (rows, blocks) or (blocks > 1 and rows > 0 and t.stride(1) != 1):
        _refuse("%s must be %d x %d with contiguous rows" % (name, rows, blocks))
    if rows > 1 and t.stride(0) < blocks:
        _refuse("the rows of %s overlap" % name)
    if t.get_device() != device:
        _refuse("%s is on another device" % name)
    return t.data_ptr(), t.stride(0) if rows > 1 else blocks


def _stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _room(workspace, nbytes, device):
    """(tensor to hold on to, address, bytes) of a call's workspace."""
    if workspace is None:
        if nbytes == 0:
            return None, None, 0
        workspace = _workspace(nbytes, torch.device("cuda", device))
    elif not workspace.is_cuda or not workspace.is_contiguous() or workspace.dtype != torch.uint8 or workspace.get_device() != device:
        _refuse("the workspace must be a contiguous uint8 tensor on the device", 5)
    return workspace, workspace.data_ptr(), workspace.numel()


def _ptr(t):
    return None if t is None else t.data_ptr()


def rms_norm(x, weight=None, eps: float = 1e-6, residual=None, quantize: bool = False, want_sum: bool = False,
             want_rstd: bool = False) -> RmsNorm:
    """h = x + residual, y = h * rstd * weight with rstd = (mean h^2 + eps)^(-1/2) of each row.  quantize: y in 8 bits with
    scales.  want_sum: h too, rounded to x's type; want_rstd: what rms_norm_backward takes."""
    rows, d, ld, dtype, device = _first("x", x)
    ld_r = 0 if residual is None else _other("residual", residual, rows, d, dtype, device)
    w = _vector("weight", weight, d, dtype, device)
    scale = rstd = total = None
    blocks = -(-d // _BLOCK)
    if quantize:
        y = x.new_empty((rows, d), dtype=_E4M3)
        scale = x.new_empty((rows, blocks), dtype=_E8M0)
    else:
        y = x.new_empty((rows, d))
    if want_sum:
        total = x.new_empty((rows, d))
    if want_rstd:
        rstd = x.new_empty(rows, dtype=_F32)
    code = _CODES[dtype]
    status = load_library().rcd_rms_norm(
        x.data_ptr(), code, rows, d, ld, _ptr(residual), ld_r, w, eps, _ptr(total), d, y.data_ptr(), 2 if quantize else code, d,
        _ptr(scale), blocks, _ptr(rstd), _stream(device))
    if status:
        _check(status)
    return RmsNorm(y, scale, total, rstd)


def rms_norm_backward(dy, h, rstd, weight=None, dsum=None, want_dweight: bool = True, workspace=None):
    """(dx, dweight) of rms_norm: h is its sum (x itself without a residual), rstd its rstd, dsum the gradient that reaches
    h along the residual stream.  dx is the residual's gradient too; dweight is None unless wanted."""
    lib = load_library()
    rows, d, ld, dtype, device = _first("dy", dy)
    ld_h = _other("h", h, rows, d, dtype, device)
    if rstd is None:
        _refuse("rstd is missing")
    r, w = _vector("rstd", rstd, rows, _F32, device), _vector("weight", weight, d, dtype, device)
    ld_s = 0 if dsum is None else _other("dsum", dsum, rows, d, dtype, device)
    dx = dy.new_empty((rows, d))
    dweight = dy.new_empty(d) if want_dweight else None
    held, room, nbytes = _room(workspace, lib.rcd_rms_norm_backward_workspace_bytes(rows, d) if want_dweight else 0, device)
    status = lib.rcd_rms_norm_backward(
        dy.data_ptr(), _CODES[dtype], rows, d, ld, h.data_ptr(), ld_h, r, w, _ptr(dsum), ld_s, dx.data_ptr(), d, _ptr(dweight), room,
        nbytes, _stream(device))
    if status:
        _check(status)
    return dx, dweight


def quantize_mxfp8(x):
    """(float8_e4m3fn elements, float8_e8m0fnu scales) of the rows of x."""
    rows, d, ld, dtype, device = _first("x", x)
    blocks = -(-d // _BLOCK)
    q, scale = x.new_empty((rows, d), dtype=_E4M3), x.new_empty((rows, blocks), dtype=_E8M0)
    _check(load_library().rcd_quantize_mxfp8(x.data_ptr(), _CODES[dtype], rows, d, ld, q.data_ptr(), d, scale.data_ptr(), blocks,
                                             _stream(device)))
    return q, scale


def _result(name, a, dtype, out_dtype, out, rows, cols, device):
    """(tensor, its type, leading dimension) of a product's result."""
    if out_dtype is None:
        out_dtype = (_BF16 if dtype is _E4M3 else dtype) if out is None else getattr(out, "dtype", None)
    if out_dtype is not _F32 and out_dtype is not _BF16:
        _refuse("the result must be float32 or bfloat16", _UNSUPPORTED)
    if out is None:
        return a.new_empty((rows, cols), dtype=out_dtype), out_dtype, cols
    return out, out_dtype, _other("out", out, rows, cols, out_dtype, device)


def linear(a, w, bias=None, act: str = "none", residual=None, a_scale=None, w_scale=None, out_dtype=None,
           want_preact: bool = False, out=None, workspace=None):
    """act(a w^T + bias) + residual, a (M, K), w (N, K).  out may be the residual.  want_preact: (y, z), z = a w^T + bias in
    float32, what linear_backward takes."""
    lib = load_library()
    M, K, ld_a, dtype, device = _first("a", a)
    ld_w = _other("w", w, None, K, dtype, device)
    N = w.shape[0]
    sa, ld_sa = _scale("a_scale", a_scale, dtype, M, K, device)
    sw, ld_sw = _scale("w_scale", w_scale, dtype, N, K, device)
    y, dt, ld_y = _result("out", a, dtype, out_dtype, out, M, N, device)
    b = _vector("bias", bias, N, dt, device)
    ld_r = 0 if residual is None else _other("residual", residual, M, N, dt, device)
    z = a.new_empty((M, N), dtype=_F32) if want_preact else None
    code = _CODES[dtype]
    held, room, nbytes = _room(workspace, lib.rcd_linear_workspace_bytes(M, N, K, code), device)
    status = lib.rcd_linear(
        a.data_ptr(), sa, ld_a, ld_sa, w.data_ptr(), sw, ld_w, ld_sw, code, _CODES[dt], M, N, K, b, _act(act), _ptr(residual), ld_r,
        _ptr(z), N, y.data_ptr(), ld_y, room, nbytes, _stream(device))
    if status:
        _check(status)
    return (y, z) if want_preact else y


def linear_backward(dy, a, w, preact=None, act: str = "none", want_da: bool = True, want_dw: bool = True, want_dbias: bool = True,
                    workspace=None):
    """(da, dw, dbias) of linear; preact is its z (not needed for act "none"); what is not wanted is None.  The residual's
    gradient is dy itself."""
    lib = load_library()
    M, N, ld_dy, dtype, device = _first("dy", dy)
    if not isinstance(a, torch.Tensor) or a.dim() != 2:
        _refuse("a must be a matrix")
    K = a.shape[1]
    ld_a, ld_w = _other("a", a, M, K, dtype, device), _other("w", w, N, K, dtype, device)
    if preact is None and act != "none":
        _refuse("preact is missing")
    ld_z = 0 if preact is None else _other("preact", preact, M, N, _F32, device)
    da = dy.new_empty((M, K)) if want_da else None
    dw = dy.new_empty((N, K)) if want_dw else None
    db = dy.new_empty(N) if want_dbias else None
    code = _CODES[dtype]
    held, room, nbytes = _room(workspace, lib.rcd_linear_backward_workspace_bytes(M, N, K, code), device)
    status = lib.rcd_linear_backward(
        dy.data_ptr(), ld_dy, a.data_ptr(), ld_a, w.data_ptr(), ld_w, code, M, N, K, _ptr(preact), ld_z, _act(act), _ptr(da), K,
        _ptr(dw), K, _ptr(db), room, nbytes, _stream(device))
    if status:
        _check(status)
    return da, dw, db


def gated_linear(a, w_gate, w_up, act: str = "silu", a_scale=None, gate_scale=None, up_scale=None, out_dtype=None,
                 want_saved: bool = False, out=None, workspace=None):
    """act(a w_gate^T) * (a w_up^T), a (M, K), both weights (F, K).  want_saved: (h, saved), saved (M, F, 2) in float32 what
    gated_linear_backward takes."""
    lib = load_library()
    M, K, ld_a, dtype, device = _first("a", a)
    ld_g = _other("w_gate", w_gate, None, K, dtype, device)
    F = w_gate.shape[0]
    ld_u = _other("w_up", w_up, F, K, dtype, device)
    sa, ld_sa = _scale("a_scale", a_scale, dtype, M, K, device)
    sg, ld_sg = _scale("gate_scale", gate_scale, dtype, F, K, device)
    su, ld_su = _scale("up_scale", up_scale, dtype, F, K, device)
    h, dt, ld_h = _result("out", a, dtype, out_dtype, out, M, F, device)
    saved = a.new_empty((M, F, 2), dtype=_F32) if want_saved else None
    code = _CODES[dtype]
    held, room, nbytes = _room(workspace, lib.rcd_gated_linear_workspace_bytes(M, F, K, code), device)
    status = lib.rcd_gated_linear(
        a.data_ptr(), sa, ld_a, ld_sa, w_gate.data_ptr(), sg, ld_g, ld_sg, w_up.data_ptr(), su, ld_u, ld_su, code, _CODES[dt], M, F,
        K, _act(act), _ptr(saved), h.data_ptr(), ld_h, room, nbytes, _stream(device))
    if status:
        _check(status)
    return (h, saved) if want_saved else h


def gated_linear_backward(dh, a, w_gate, w_up, saved, act: str = "silu", want_da: bool = True, want_dw: bool = True,
                          workspace=None):
    """(da, dw_gate, dw_up) of gated_linear; saved is its saved; what is not wanted is None."""
    lib = load_library()
    M, F, ld_dh, dtype, device = _first("dh", dh)
    if not isinstance(a, torch.Tensor) or a.dim() != 2:
        _refuse("a must be a matrix")
    K = a.shape[1]
    ld_a = _other("a", a, M, K, dtype, device)
    ld_g, ld_u = _other("w_gate", w_gate, F, K, dtype, device), _other("w_up", w_up, F, K, dtype, device)
    if (not isinstance(saved, torch.Tensor) or saved.shape != (M, F, 2) or saved.dtype is not _F32
            or not saved.is_contiguous() or saved.get_device() != device):
        _refuse("saved must be what gated_linear returned")
    da = dh.new_empty((M, K)) if want_da else None
    dwg = dh.new_empty((F, K)) if want_dw else None
    dwu = dh.new_empty((F, K)) if want_dw else None
    code = _CODES[dtype]
    held, room, nbytes = _room(workspace, lib.rcd_gated_linear_backward_workspace_bytes(M, F, K, code), device)
    status = lib.rcd_gated_linear_backward(
        dh.data_ptr(), ld_dh, a.data_ptr(), ld_a, w_gate.data_ptr(), ld_g, w_up.data_ptr(), ld_u, code, M, F, K, saved.data_ptr(),
        _act(act), _ptr(da), K, _ptr(dwg), K, _ptr(dwu), K, room, nbytes, _stream(device))
    if status:
        _check(status)
    return da, dwg, dwu
