"""ctypes binding of the operators from the residual stream to log probabilities (rms_norm.h, token_logp.h, fp8_blocks.h): argument
marshalling only, same names as the C entry points, and the front ends ``rms_norm`` and ``token_log_probs`` (torch.autograd),
``rms_norm_fp8``, ``quantize_blocks_fp8`` and ``token_log_probs_fp8``.

As in the other bindings, the functions check device, dtype, shape and contiguity, pass raw device pointers and the current stream,
and turn non-zero status codes into ``VpceError``.  There is no CPU or PyTorch fallback.  The gradients have no derivative of
their own: differentiating them again raises.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple, Union

import torch

from .autograd import _pick_chunk, _workspace as _ce_workspace, first_derivative_only
from .binding import load_library
from .training_ops import _BF16, _DTYPE_CODE, _F32, _call, _device, _fail, _opt, _ptr, _rows, _stream, _workspace

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
            "vp_token_logp_workspace_bytes": (sz, [i64, i64, i64, i32]),
            "vp_token_logp_forward": (i32, [vp, vp, vp, i64, i64, i64, f64, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp]),
            "vp_token_logp_backward": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, f64, i64, i32, i64, i64, i32, vp, sz, vp]),
            "vp_token_logp_debug_drop": (i32, [i32]),
            "vp_token_logp_fp8_workspace_bytes": (sz, [i64, i64, i64, i32]),
            "vp_token_logp_fp8_forward": (i32, [vp, vp, vp, vp, vp, i64, i64, i64, f64, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp]),
            "vp_fp8_quantize_blocks": (i32, [vp, i32, i64, i64, i64, vp, i64, vp, vp]),
        }
        for name, (res, args) in signatures.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _LIB = lib
    return _LIB


def fp8_blocks(n: int) -> int:
    """Blocks of 128 that n rows or columns fall into."""
    return -(-n // FP8_BLOCK)


def _matrix(t, dtype, name: str, rows: int, cols: int, dev: int) -> int:
    """Pointer of a contiguous [rows, cols] tensor: as many elements in another shape are in another order."""
    p = _ptr(t, dtype, name, rows * cols, dev)
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must be [{rows}, {cols}], got {list(t.shape)}")
    return p


def _opt_matrix(t, dtype, name: str, rows: int, cols: int, dev: int) -> Optional[int]:
    return None if t is None else _matrix(t, dtype, name, rows, cols, dev)


# --------------------------------------------------------------------------- RMS norm (rms_norm.h)
def _rms_types(dt, weight):
    """The weight's element type, checked against the rows' type dt."""
    if dt not in _DTYPE_CODE:
        raise TypeError(f"x must be bfloat16, float16 or float32, got {dt}")
    wdt = dt if weight is None else weight.dtype
    if wdt is not dt and wdt is not _F32:
        raise TypeError(f"weight and its gradient must be {dt} or float32, got {wdt}")
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
    dt = x.dtype
    wdt = _rms_types(dt, weight)
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
    _call(_lib().vp_rms_forward_fp8, dev, *head, eps, qp, qs, _matrix(scales, _F32, "scales", rows, fp8_blocks(d), dev), *tail,
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
    dt = z.dtype
    wdt = _rms_types(dt, dweight if weight is None else weight)
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
        vp_rms_forward(x2, r2, weight, eps, y.view(x2.shape), None if z is None else z.view(x2.shape), rstd)
        # the sum as it is returned: a saved view of it would hold its own node, which nothing frees without a backward pass
        ctx.save_for_backward(x2 if z is None else z, weight, rstd)
        ctx.shape = x.shape
        ctx.set_materialize_grads(False)
        return y if z is None else (y, z)

    @staticmethod
    @first_derivative_only
    def backward(ctx, dy, dz=None):
        z, weight, rstd = ctx.saved_tensors
        z = z.reshape(-1, z.shape[-1])
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
                       q.view(x2.shape), scales.view(x2.shape[0], fp8_blocks(d)), None if z is None else z.view(x2.shape), None)
    return (q, scales) if z is None else (q, scales, z)


# --------------------------------------------------------------------------- quantisation in blocks (fp8_blocks.h)
def vp_fp8_quantize_blocks(w, q, scales, stream=None) -> None:
    """q [rows, d] float8_e4m3fn and scales [ceil(rows / 128), ceil(d / 128)] float32 of the weight w [rows, d], w = q * scale.  See
    include/fp8_blocks.h."""
    dev = _device(w, "w")
    if w.dim() != 2 or w.dtype not in _DTYPE_CODE:
        raise TypeError(f"w must be [rows, d] in bfloat16, float16 or float32, got {list(w.shape)} {w.dtype}")
    rows, d = w.shape
    wp, ws = _rows(w, w.dtype, "w", rows, d, dev)
    qp, qs = _rows(q, _F8, "q", rows, d, dev)
    _call(_lib().vp_fp8_quantize_blocks, dev, wp, _DTYPE_CODE[w.dtype], rows, d, ws, qp, qs,
          _matrix(scales, _F32, "scales", fp8_blocks(rows), fp8_blocks(d), dev), _stream(stream, dev))


def quantize_blocks_fp8(w: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(q, scales) of a weight [rows, d]: float8_e4m3fn and one float32 scale for each 128 x 128 block, w = q * scale.

    What ``token_log_probs_fp8`` takes as its weight.  There is no gradient."""
    _device(w, "w")
    if w.dim() != 2:
        raise ValueError(f"w must be [rows, d], got {list(w.shape)}")
    w = w.detach()
    rows, d = w.shape
    w = _as_rows(w, d)
    q = torch.empty(rows, d, dtype=_F8, device=w.device)
    scales = torch.empty(fp8_blocks(rows), fp8_blocks(d), dtype=_F32, device=w.device)
    vp_fp8_quantize_blocks(w, q, scales)
    return q, scales


# --------------------------------------------------------------------------- token log probabilities (token_logp.h)
MAX_TOP = 20                                               # alternatives per token
GRAD_TEMPERATURES = (0.01, 100.0)                          # of the backward pass; the forward pass takes 1e-6 to 1e6

_I32 = torch.int32
_TOKEN_TYPES = frozenset((torch.uint8, torch.int8, torch.int16, torch.int32, torch.int64))


def vp_token_logp_workspace_bytes(T: int, d: int, V: int, top: int) -> int:
    return _lib().vp_token_logp_workspace_bytes(T, d, V, top)


def vp_token_logp_fp8_workspace_bytes(T: int, d: int, V: int, top: int) -> int:
    return _lib().vp_token_logp_fp8_workspace_bytes(T, d, V, top)


def _head_shapes(H, W, h: str, w: str):
    dev = _device(H, h)
    _device(W, w)
    if H.dim() != 2 or W.dim() != 2 or H.shape[1] != W.shape[1]:
        raise ValueError(f"{h} must be [T, d] and {w} [V, d], got {list(H.shape)} and {list(W.shape)}")
    return dev, H.shape[0], H.shape[1], W.shape[0]


def _logp_outputs(dev, T, tokens, logp, lse, entropy, top_logp, top_ids):
    if (tokens is None) != (logp is None):
        raise ValueError("tokens and logp go together")
    if (top_logp is None) != (top_ids is None):
        raise ValueError("top_logp and top_ids go together")
    top = 0
    if top_logp is not None:
        if top_logp.dim() != 2 or top_logp.shape[0] != T:
            raise ValueError(f"top_logp must be [{T}, alternatives], got {list(top_logp.shape)}")
        top = top_logp.shape[1]
    return top, (_opt(logp, _F32, "logp", T, dev), _opt(lse, _F32, "lse", T, dev), _opt(entropy, _F32, "entropy", T, dev),
                 _opt_matrix(top_logp, _F32, "top_logp", T, top, dev), _opt_matrix(top_ids, _I32, "top_ids", T, top, dev), top)


def vp_token_logp_forward(H, W, tokens, temperature: float, ignore_index: int, logp, lse, entropy, top_logp, top_ids, workspace,
                          stream=None) -> None:
    """logp, lse, entropy [T] and the alternatives top_logp, top_ids [T, top] of H [T, d] and W [V, d] (bfloat16) at the given tokens
    [T] (int32).  tokens and logp, lse, entropy, top_logp and top_ids may be None.  See include/token_logp.h."""
    dev, T, d, V = _head_shapes(H, W, "H", "W")
    top, outs = _logp_outputs(dev, T, tokens, logp, lse, entropy, top_logp, top_ids)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_token_logp_forward, dev, _ptr(H, _BF16, "H", T * d, dev), _ptr(W, _BF16, "W", V * d, dev),
          _opt(tokens, _I32, "tokens", T, dev), T, d, V, temperature, ignore_index, *outs, wsp, wsn, _stream(stream, dev))


def vp_token_logp_fp8_forward(Hq, Hs, Wq, Ws, tokens, temperature: float, ignore_index: int, logp, lse, entropy, top_logp, top_ids,
                              workspace, stream=None) -> None:
    """The same from 8-bit operands: Hq [T, d] and Wq [V, d] float8_e4m3fn with their float32 scales Hs [T, ceil(d / 128)] and Ws
    [ceil(V / 128), ceil(d / 128)].  See include/token_logp.h."""
    dev, T, d, V = _head_shapes(Hq, Wq, "Hq", "Wq")
    top, outs = _logp_outputs(dev, T, tokens, logp, lse, entropy, top_logp, top_ids)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_token_logp_fp8_forward, dev, _ptr(Hq, _F8, "Hq", T * d, dev), _matrix(Hs, _F32, "Hs", T, fp8_blocks(d), dev),
          _ptr(Wq, _F8, "Wq", V * d, dev), _matrix(Ws, _F32, "Ws", fp8_blocks(V), fp8_blocks(d), dev), _opt(tokens, _I32, "tokens", T, dev), T, d,
          V, temperature, ignore_index, *outs, wsp, wsn, _stream(stream, dev))


def vp_token_logp_backward(H, W, tokens, lse, entropy, dlogp, dent, temperature: float, ignore_index: int, dH, dW, block_v: int, T_chunk: int,
                           accumulate_dW: bool, workspace, chunk_index_base: int = 0, stream=None) -> None:
    """dH [T, d] (bfloat16) and dW [V, d] (float32, overwritten or added to) from the upstream gradients dlogp and dent [T] (one of
    them may be None, as may dH or dW) and the forward call's lse and entropy (the latter with dent only).  temperature: 0.01 to 100.
    workspace: vp_ce_workspace_bytes(T_chunk, d, block_v).  See include/token_logp.h."""
    dev, T, d, V = _head_shapes(H, W, "H", "W")
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_token_logp_backward, dev, _ptr(H, _BF16, "H", T * d, dev), _ptr(W, _BF16, "W", V * d, dev),
          _ptr(tokens, _I32, "tokens", T, dev), _ptr(lse, _F32, "lse", T, dev), _opt(entropy, _F32, "entropy", T, dev),
          _opt(dlogp, _F32, "dlogp", T, dev), _opt(dent, _F32, "dent", T, dev), _opt_matrix(dH, _BF16, "dH", T, d, dev),
          _opt_matrix(dW, _F32, "dW", V, d, dev), T, d, V, temperature, block_v, ignore_index, T_chunk, chunk_index_base, 1 if accumulate_dW else 0,
          wsp, wsn, _stream(stream, dev))


def vp_token_logp_debug_drop(k_block: int) -> None:
    """Test hook: the next forward launch loses the copies of one k-block (see include/token_logp.h); < 0 disarms."""
    code = _lib().vp_token_logp_debug_drop(k_block)
    if code:
        _fail(code)


class TokenLogProbs(NamedTuple):
    """Log probability of each given token (None without tokens), entropy of its distribution, and the alternatives' log
    probabilities and ids [T, top_k] (None where top_k is 0)."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


def _check_top(top_k: int, V: int) -> int:
    top_k = int(top_k)
    if not 0 <= top_k <= min(MAX_TOP, V):
        raise ValueError(f"top_k must lie between 0 and {min(MAX_TOP, V)}, got {top_k}")
    return top_k


def _as_tokens(tokens) -> Optional[torch.Tensor]:
    """tokens as contiguous int32; a number that 32 bits do not hold stays outside every vocabulary."""
    if tokens is None:
        return None
    if not isinstance(tokens, torch.Tensor) or tokens.dtype not in _TOKEN_TYPES:
        raise TypeError(f"tokens must be a tensor of integers, got {getattr(tokens, 'dtype', type(tokens))}")
    if tokens.dtype is torch.int64:
        tokens = tokens.clamp(-1 << 31, (1 << 31) - 1)
    return tokens.to(_I32).contiguous()


def _check_ignore_index(ignore_index) -> int:
    ignore_index = int(ignore_index)
    if not -1 << 31 <= ignore_index < 1 << 31:
        raise ValueError(f"ignore_index must fit 32 bits, got {ignore_index}")
    return ignore_index


def _empty_outputs(T: int, top: int, tokens, device):
    f32 = lambda *shape: torch.empty(*shape, dtype=_F32, device=device)  # noqa: E731
    return (None if tokens is None else f32(T), f32(T), f32(T), f32(T, top) if top else None,
            torch.empty(T, top, dtype=_I32, device=device) if top else None)


def _strip_width(T_chunk: int, V: int) -> int:
    """Columns of the vocabulary that the backward pass has under way at once where the caller does not say: 16384, or 8192 where a chunk
    has more than 8192 tokens, in whole tiles.

    A strip's part of dH is one sum of the tensor core, which cuts off up to 2^-23 of what it holds for every 16 columns; parts are
    added in fp32.  Wider strips save launches and passes over dH's sums, but where rows of W have a common mean (1, of a spread of 0.1; 201088
    x 640, 200 tokens) dH is off by 1.79e-3 (Frobenius) with 8192 columns, 1.84e-3 with 16384, 2.03e-3 with 32768 and 5.5e-3 with all, of which
    the rounding to bf16 is 1.64e-3.  201088 x 2880, backward: 200 tokens 3.0 ms with 8192 columns, 2.4 with 16384, 1.8 with all; 1000
    tokens 5.1, 4.1 and 3.9; 8192 tokens 24.8 and 24.2."""
    return min(16384 if T_chunk <= 8192 else 8192, -(-V // 256) * 256)


class _TokenLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, H, W, tokens, top, temperature, ignore_index, block_v, T_chunk, dW_accum):
        H, W = H.contiguous(), W.contiguous()
        tokens = _as_tokens(tokens)
        T, d = H.shape
        logp, lse, entropy, top_logp, top_ids = _empty_outputs(T, top, tokens, H.device)
        n = vp_token_logp_workspace_bytes(T, d, W.shape[0], top)
        if n == 0:
            raise ValueError(f"unsupported shape: d must be a multiple of 8, got {d}")
        vp_token_logp_forward(H, W, tokens, temperature, ignore_index, logp, lse, entropy, top_logp, top_ids,
                              torch.empty(n, dtype=torch.uint8, device=H.device))
        ctx.save_for_backward(H, W, tokens, lse, entropy)
        ctx.cfg = (temperature, ignore_index, block_v, T_chunk)
        ctx.dW_accum = dW_accum
        ctx.set_materialize_grads(False)
        if top:
            ctx.mark_non_differentiable(top_logp, top_ids)
        return logp, entropy, top_logp, top_ids

    @staticmethod
    @first_derivative_only
    def backward(ctx, dlogp, dent, _top_logp, _top_ids):
        H, W, tokens, lse, entropy = ctx.saved_tensors
        temperature, ignore_index, block_v, T_chunk = ctx.cfg
        accum = ctx.dW_accum
        need_dH, need_dW = ctx.needs_input_grad[0], accum is not None or ctx.needs_input_grad[1]
        if not (need_dH or need_dW) or (dlogp is None and dent is None):
            return (None,) * 9
        if not GRAD_TEMPERATURES[0] <= temperature <= GRAD_TEMPERATURES[1]:
            raise ValueError(f"gradients need a temperature between {GRAD_TEMPERATURES[0]} and {GRAD_TEMPERATURES[1]}, got {temperature}")
        T, d = H.shape
        T_chunk = _pick_chunk(T, T_chunk)
        if block_v is None:
            block_v = _strip_width(T_chunk, W.shape[0])
        ws = _ce_workspace(T_chunk, d, block_v, H.device)
        dH = torch.empty_like(H) if need_dH else None
        dW = None
        if need_dW:
            dW = accum if accum is not None else torch.empty(W.shape, dtype=_F32, device=W.device)
        if tokens is None:
            tokens = torch.full((T,), ignore_index, dtype=_I32, device=H.device)
        grads = [None if g is None else g.to(_F32).contiguous() for g in (dlogp, dent)]
        vp_token_logp_backward(H, W, tokens, lse, entropy, *grads, temperature, ignore_index, dH, dW, block_v, T_chunk, accum is not None, ws)
        # with an fp32 accumulation buffer the weight gradient lives there (main-grad style); autograd gets none
        grad_W = None if (accum is not None or dW is None) else dW.to(W.dtype)
        return (dH, grad_W) + (None,) * 7


def token_log_probs(H: torch.Tensor, W: torch.Tensor, tokens: Optional[torch.Tensor] = None, top_k: int = 0, temperature: float = 1.0,
                    ignore_index: int = -100, block_v: Optional[int] = None, T_chunk: Optional[int] = None,
                    dW_accum: Optional[torch.Tensor] = None) -> TokenLogProbs:
    """Log probabilities of ``tokens`` under softmax(H @ W.T / temperature), with entropy and ``top_k`` alternatives.

    H ``[T, d]`` and W ``[V, d]`` are bfloat16 CUDA tensors, ``tokens`` ``[T]`` integers of 8 to 64 bits (``ignore_index``, or any number
    outside the vocabulary: logp 0, no gradient of it), or None where only entropy and alternatives are asked for.  logp and entropy are
    differentiable in H and W (temperatures from 0.01 to 100; without gradients 1e-6 to 1e6); the logits are never materialised.
    Alternatives come larger first, among equals the lower id; at most 20.  ``block_v`` (None: 16384, or 8192 where a chunk has more than
    8192 tokens) and ``T_chunk`` (None: up to 16384) are the backward pass's, which holds T_chunk x block_v elements of bf16 at once, as is
    ``dW_accum`` (float32 ``[V, d]``: the weight gradient is added into it and ``W.grad`` stays untouched); see
    ``vocab_proj_cross_entropy``.  The device status word is left unread, as there: who has to know of tokens outside the vocabulary
    calls ``vp_token_logp_forward`` with a workspace and ``vp_ce_device_status``; after a wait that ran out the results are NaN."""
    _, _, _, V = _head_shapes(H, W, "H", "W")
    if H.dtype is not _BF16 or W.dtype is not _BF16:
        raise TypeError("H and W must be bfloat16 CUDA tensors")
    return TokenLogProbs(*_TokenLogProbs.apply(H, W, tokens, _check_top(top_k, V), float(temperature), _check_ignore_index(ignore_index),
                                               None if block_v is None else int(block_v), T_chunk, dW_accum))


def token_log_probs_fp8(Hq: torch.Tensor, Hs: torch.Tensor, Wq: torch.Tensor, Ws: torch.Tensor, tokens: Optional[torch.Tensor] = None,
                        top_k: int = 0, temperature: float = 1.0, ignore_index: int = -100) -> TokenLogProbs:
    """``token_log_probs`` from 8-bit operands, without a gradient: for scoring and generation.

    Hq ``[T, d]`` with Hs ``[T, ceil(d / 128)]`` is what ``rms_norm_fp8`` returns, Wq ``[V, d]`` with Ws what ``quantize_blocks_fp8``
    returns.  There is no gradient: under ``torch.no_grad()``, or with scales that require none."""
    _, T, d, V = _head_shapes(Hq, Wq, "Hq", "Wq")
    if torch.is_grad_enabled() and (Hs.requires_grad or Ws.requires_grad):
        raise RuntimeError("token_log_probs_fp8 has no gradient: call it under torch.no_grad()")
    top = _check_top(top_k, V)
    tokens, ignore_index = _as_tokens(tokens), _check_ignore_index(ignore_index)
    logp, lse, entropy, top_logp, top_ids = _empty_outputs(T, top, tokens, Hq.device)
    n = vp_token_logp_fp8_workspace_bytes(T, d, V, top)
    if n == 0:
        raise ValueError(f"unsupported shape: d must be a multiple of 16, at most 16384, got {d}")
    vp_token_logp_fp8_forward(Hq.contiguous(), Hs.contiguous(), Wq.contiguous(), Ws.contiguous(), tokens, float(temperature), ignore_index, logp,
                              lse, entropy, top_logp, top_ids, torch.empty(n, dtype=torch.uint8, device=Hq.device))
    return TokenLogProbs(logp, entropy, top_logp, top_ids)
