"""ctypes binding of the operators from the residual stream to log probabilities (rms_norm.h): argument marshalling only, same
names as the C entry points, and the front ends ``rms_norm`` (torch.autograd) and ``rms_norm_fp8``.

As in the other bindings, the functions check device, dtype, shape and contiguity, pass raw device pointers and the current stream,
and turn non-zero status codes into ``VpceError``.  There is no CPU or PyTorch fallback.  The gradients have no derivative of
their own: differentiating them again raises.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple, Union

import torch

from .autograd import first_derivative_only
from .binding import load_library
from .training_ops import _DTYPE_CODE, _F32, _call, _device, _opt, _ptr, _rows, _stream, _workspace

_F8 = torch.float8_e4m3fn
FP8_BLOCK = 128                                            # columns (and rows of a weight) that share a scale

_LIB: Optional[ctypes.CDLL] = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        lib = load_library()
        i64, i32, vp, sz, f64 = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double
        signatures = {
            "vp_rms_forward": (i32, [vp, i32, i64, i64, i64, vp, i64, vp, i32, f64, vp, i64, vp, i64, vp, vp]),
            "vp_rms_forward_fp8": (i32, [vp, i32, i64, i64, i64, vp, i64, vp, i32, f64, vp, i64, vp, vp, i64, vp, vp]),
            "vp_rms_workspace_bytes": (sz, [i64, i64]),
            "vp_rms_backward": (i32, [vp, i64, vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, i64, vp, vp, sz, vp]),
        }
        for name, (res, args) in signatures.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _LIB = lib
    return _LIB


def fp8_blocks(n: int) -> int:
    """Blocks of 128 that n rows or columns fall into."""
    return -(-n // FP8_BLOCK)


# --------------------------------------------------------------------------- RMS norm (rms_norm.h)
def _rms_types(x, *weights):
    if x.dtype not in _DTYPE_CODE:
        raise TypeError(f"x must be bfloat16, float16 or float32, got {x.dtype}")
    wdt = next((w.dtype for w in weights if w is not None), x.dtype)
    if wdt is not x.dtype and wdt is not _F32:
        raise TypeError(f"weight and its gradient must be {x.dtype} or float32, got {wdt}")
    return wdt


def _opt_rows(t, dtype, name: str, rows: int, d: int, dev: int):
    return (None, d) if t is None else _rows(t, dtype, name, rows, d, dev)


def _rms_inputs(x, residual, weight, z, rstd):
    dev = _device(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    if residual is None and z is not None:
        raise ValueError("z is the sum with a residual: without one it is x itself")
    rows, d = x.shape
    wdt, dt = _rms_types(x, weight), x.dtype
    xp, xs = _rows(x, dt, "x", rows, d, dev)
    rp, rs = _opt_rows(residual, dt, "residual", rows, d, dev)
    zp, zs = _opt_rows(z, dt, "z", rows, d, dev)
    head = (xp, _DTYPE_CODE[dt], rows, d, xs, rp, rs, _opt(weight, wdt, "weight", d, dev), _DTYPE_CODE[wdt])
    return dev, rows, d, head, (zp, zs, _opt(rstd, _F32, "rstd", rows, dev))


def vp_rms_forward(x, residual, weight, eps: float, y, z, rstd, stream=None) -> None:
    """z = x + residual (rounded; x itself where residual is None), y = z / rms(z) * weight per row of x [rows, d].  z, rstd [rows]
    float32, residual and weight may be None.  See include/rms_norm.h."""
    dev, rows, d, head, tail = _rms_inputs(x, residual, weight, z, rstd)
    yp, ys = _rows(y, x.dtype, "y", rows, d, dev)
    _call(_lib().vp_rms_forward, dev, *head, eps, yp, ys, *tail, _stream(stream, dev))


def vp_rms_forward_fp8(x, residual, weight, eps: float, q, scales, z, rstd, stream=None) -> None:
    """The same with y in 8 bits: q [rows, d] float8_e4m3fn and scales [rows, ceil(d / 128)] float32, y = q * scale.  See
    include/rms_norm.h."""
    dev, rows, d, head, tail = _rms_inputs(x, residual, weight, z, rstd)
    qp, qs = _rows(q, _F8, "q", rows, d, dev)
    _call(_lib().vp_rms_forward_fp8, dev, *head, eps, qp, qs, _ptr(scales, _F32, "scales", rows * fp8_blocks(d), dev), *tail,
          _stream(stream, dev))


def vp_rms_workspace_bytes(rows: int, d: int) -> int:
    return _lib().vp_rms_workspace_bytes(rows, d)


def vp_rms_backward(dy, dz, z, weight, rstd, dx, dweight, workspace, stream=None) -> None:
    """dx [rows, d] (the residual's gradient, too) and dweight [d] (each may be None: not computed) from the upstream gradients dy of
    y and dz of z (None: zeros) and the forward call's z (x where there was no residual) and rstd.  workspace (uint8) is needed for
    dweight only.  See include/rms_norm.h."""
    dev = _device(z, "z")
    if z.dim() != 2:
        raise ValueError("z must be [rows, d]")
    rows, d = z.shape
    wdt, dt = _rms_types(z, weight, dweight), z.dtype
    zp, zs = _rows(z, dt, "z", rows, d, dev)
    dyp, dys = _rows(dy, dt, "dy", rows, d, dev)
    dzp, dzs = _opt_rows(dz, dt, "dz", rows, d, dev)
    dxp, dxs = _opt_rows(dx, dt, "dx", rows, d, dev)
    wsp, wsn = (None, 0) if workspace is None else _workspace(workspace, dev)
    _call(_lib().vp_rms_backward, dev, dyp, dys, dzp, dzs, zp, zs, _DTYPE_CODE[dt], rows, d, _opt(weight, wdt, "weight", d, dev),
          _DTYPE_CODE[wdt], _ptr(rstd, _F32, "rstd", rows, dev), dxp, dxs, _opt(dweight, wdt, "dweight", d, dev), wsp, wsn,
          _stream(stream, dev))


def _as_rows(t, d: int):
    """t as [rows, d] with contiguous rows that do not overlap; a copy where its strides do not allow it."""
    t = t.reshape(-1, d)
    return t.contiguous() if t.stride(-1) != 1 or (t.shape[0] > 1 and t.stride(0) < d) else t


def _check_norm_input(x, residual) -> None:
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must have a last dimension of at least 1")
    if residual is not None and residual.shape != x.shape:
        raise ValueError(f"residual must have x's shape {list(x.shape)}, got {list(residual.shape)}")


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        d = x.shape[-1]
        x2 = _as_rows(x, d)
        r2 = None if residual is None else _as_rows(residual, d)
        weight = None if weight is None else weight.contiguous()
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        z = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(x2.shape[0], dtype=_F32, device=x.device)
        z2 = x2 if z is None else z.view(x2.shape)
        vp_rms_forward(x2, r2, weight, eps, y.view(x2.shape), None if z is None else z2, rstd)
        ctx.save_for_backward(z2, weight, rstd)
        ctx.shape = x.shape
        ctx.set_materialize_grads(False)
        return y if z is None else (y, z)

    @staticmethod
    @first_derivative_only
    def backward(ctx, dy, dz=None):
        z, weight, rstd = ctx.saved_tensors
        rows, d = z.shape
        need_x, need_w, need_r, _ = ctx.needs_input_grad
        need_w = need_w and weight is not None
        if dy is None:                                      # only the sum was used: its gradient goes on as it is
            return (dz if need_x else None), (torch.zeros_like(weight) if need_w else None), (dz if need_r else None), None
        dx = torch.empty(rows, d, dtype=z.dtype, device=z.device) if need_x or need_r else None
        dw = torch.empty_like(weight) if need_w else None
        ws = torch.empty(vp_rms_workspace_bytes(rows, d), dtype=torch.uint8, device=z.device) if need_w else None
        vp_rms_backward(_as_rows(dy, d), None if dz is None else _as_rows(dz, d), z, weight, rstd, dx, dw, ws)
        dx = None if dx is None else dx.view(ctx.shape)
        return (dx if need_x else None), dw, (dx if need_r else None), None


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
             eps: float = 1e-6) -> Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]:
    """RMS norm over the last dimension; with a residual of x's shape, of their sum: returns (y, x + residual).

    Differentiable in x, weight and residual.  x is bfloat16, float16 or float32 of any shape; weight ``[d]`` has x's dtype or
    float32.  Statistics are float32; each result is rounded once, and the norm is of the sum as it is returned."""
    _check_norm_input(x, residual)
    return _RmsNorm.apply(x, weight, residual, float(eps))


def rms_norm_fp8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                 eps: float = 1e-6) -> Tuple[torch.Tensor, ...]:
    """``rms_norm`` with its output in 8 bits: (q, scales) or, with a residual, (q, scales, x + residual).

    q is float8_e4m3fn of x's shape, scales float32 ``[..., ceil(d / 128)]``: 128 neighbouring columns share one, y = q * scale.
    There is no gradient: under ``torch.no_grad()``, or with inputs that require none."""
    _check_norm_input(x, residual)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, residual)):
        raise RuntimeError("rms_norm_fp8 has no gradient: call it under torch.no_grad()")
    d = x.shape[-1]
    x2 = _as_rows(x, d)
    q = torch.empty(x.shape, dtype=_F8, device=x.device)
    scales = torch.empty(*x.shape[:-1], fp8_blocks(d), dtype=_F32, device=x.device)
    z = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    vp_rms_forward_fp8(x2, None if residual is None else _as_rows(residual, d), None if weight is None else weight.contiguous(), float(eps),
                       q.view(x2.shape), scales, None if z is None else z.view(x2.shape), None)
    return (q, scales) if z is None else (q, scales, z)
