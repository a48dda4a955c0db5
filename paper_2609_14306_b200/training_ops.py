"""ctypes binding of the operators around the head (layer_norm.h, sequence_loss.h, muon.h): argument marshalling only,
same names as the C entry points, and the torch.autograd front ends ``layer_norm``, ``policy_loss`` and
``preference_loss``.

Like the head's binding, the functions check device, dtype, shape and contiguity, pass raw device pointers and the current
stream, and turn non-zero status codes into ``VpceError``.  There is no CPU or PyTorch fallback.  The gradients have no
derivative of their own: differentiating them again raises.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence, Tuple

import torch

from .autograd import first_derivative_only
from .binding import VpceError, load_library, vp_ce_status_string

_F32, _BF16, _F16 = torch.float32, torch.bfloat16, torch.float16
_DTYPE_CODE = {_BF16: 0, _F16: 1, _F32: 2}
_AGGREGATE = {"token_mean": 0, "seq_mean": 1}
_KIND = {"sigmoid": 0, "ipo": 1}

_LIB: Optional[ctypes.CDLL] = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        lib = load_library()
        i64, i32, vp, sz, f64 = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double
        signatures = {
            "vp_ln_forward": (i32, [vp, i32, i64, i64, i64, vp, vp, i32, f64, vp, i64, vp, vp, vp]),
            "vp_ln_workspace_bytes": (sz, [i64, i64]),
            "vp_ln_backward": (i32, [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, i64, vp, vp, vp, sz, vp]),
            "vp_policy_loss_workspace_bytes": (sz, [i64, i64]),
            "vp_policy_loss": (i32, [vp, vp, vp, vp, i32, vp, vp, i64, i64, f64, f64, f64, i32, vp, vp, vp, vp, sz, vp]),
            "vp_policy_loss_backward": (i32, [vp, vp, vp, vp, i32, vp, vp, i64, i64, f64, f64, f64, i32, vp, vp, vp, sz, vp]),
            "vp_preference_loss_workspace_bytes": (sz, [i64, i64]),
            "vp_preference_loss": (i32, [vp, vp, vp, vp, i64, i64, f64, f64, f64, i32, i32, vp, vp, vp, vp, vp, sz, vp]),
            "vp_preference_loss_backward": (i32, [vp, vp, i64, i64, vp, vp, vp, sz, vp]),
            "muon_workspace_bytes": (sz, [i64, i64, i64]),
            "muon_orthogonalize": (i32, [vp, i32, vp, i32, i64, i64, i64, vp, i32, f64, vp, sz, vp]),
            "muon_step": (i32, [vp, vp, vp, i32, vp, i64, i64, i64, f64, f64, i32, f64, f64, vp, i32, f64, vp, sz, vp]),
            "muon_device_status": (i32, [vp, ctypes.POINTER(ctypes.c_int32), vp]),
            "muon_debug_drop": (i32, [i32, i32, i32]),
        }
        for name, (res, args) in signatures.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _LIB = lib
    return _LIB


def _fail(code: int) -> None:
    raise VpceError(code, vp_ce_status_string(code))


def _stream(stream, index: int) -> int:
    """Raw cudaStream_t: the given stream, else the current stream of device `index`."""
    return int(stream.cuda_stream) if stream is not None else torch._C._cuda_getCurrentRawStream(index)


def _call(fn, index: int, *args) -> None:
    """Calls the C entry point with the operands' device current (the library launches on the current device)."""
    if torch._C._cuda_getDevice() == index:
        code = fn(*args)
    else:
        with torch.cuda.device(index):
            code = fn(*args)
    if code:
        _fail(code)


def _device(t, name: str) -> int:
    """Index of the device that holds t."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.get_device()


def _ptr(t, dtype, name: str, numel: int, dev: int) -> int:
    """Pointer of a contiguous tensor of `numel` elements on device `dev`."""
    # what is right is found out with as few calls as possible; what is wrong, and why, below
    if type(t) is torch.Tensor and t.dtype is dtype and t.numel() == numel and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{dev}")
    return t.data_ptr()


def _opt(t, dtype, name: str, numel: int, dev: int) -> Optional[int]:
    return None if t is None else _ptr(t, dtype, name, numel, dev)


def _workspace(t, dev: int) -> Tuple[int, int]:
    n = t.numel() if isinstance(t, torch.Tensor) else 0
    return _ptr(t, torch.uint8, "workspace", n, dev), n


# --------------------------------------------------------------------------- layer norm (layer_norm.h)
def _rows(t, dtype, name: str, rows: int, d: int, dev: int) -> Tuple[int, int]:
    """Pointer and row stride of a [rows, d] tensor whose rows are contiguous."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.shape == (rows, d) and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr(), d
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != d:
        raise ValueError(f"{name} must be [{rows}, {d}], got {list(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{dev}")
    s0, s1 = t.stride()
    if d > 1 and rows > 0 and s1 != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if rows <= 1:
        s0 = d
    elif s0 < d:
        raise ValueError(f"{name}: rows overlap (row stride {s0} below {d})")
    return t.data_ptr(), s0


def _ln_types(x, weight, *others):
    if x.dtype not in _DTYPE_CODE:
        raise TypeError(f"x must be bfloat16, float16 or float32, got {x.dtype}")
    wdt = x.dtype
    for w in (weight, *others):
        if w is not None:
            wdt = w.dtype
            break
    if wdt is not x.dtype and wdt is not _F32:
        raise TypeError(f"weight, bias and their gradients must be {x.dtype} or float32, got {wdt}")
    return wdt


def vp_ln_forward(x, weight, bias, eps: float, y, mean, rstd, stream=None) -> None:
    """y = (x - mean) * rstd * weight + bias per row of x [rows, d]; mean and rstd [rows] float32 (both may be None, as may
    weight and bias).  See include/layer_norm.h."""
    dev = _device(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    rows, d = x.shape
    wdt = _ln_types(x, weight, bias)
    dt = x.dtype
    xp, xs = _rows(x, dt, "x", rows, d, dev)
    yp, ys = _rows(y, dt, "y", rows, d, dev)
    _call(_lib().vp_ln_forward, dev, xp, _DTYPE_CODE[dt], rows, d, xs, _opt(weight, wdt, "weight", d, dev),
          _opt(bias, wdt, "bias", d, dev), _DTYPE_CODE[wdt], eps, yp, ys, _opt(mean, _F32, "mean", rows, dev),
          _opt(rstd, _F32, "rstd", rows, dev), _stream(stream, dev))


def vp_ln_workspace_bytes(rows: int, d: int) -> int:
    return _lib().vp_ln_workspace_bytes(rows, d)


def vp_ln_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream=None) -> None:
    """dx [rows, d], dweight [d], dbias [d] (each may be None: not computed) from the upstream gradient dy and the forward
    call's x, mean and rstd.  workspace (uint8) is needed for dweight and dbias only.  See include/layer_norm.h."""
    dev = _device(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [rows, d]")
    rows, d = x.shape
    wdt = _ln_types(x, weight, dweight, dbias)
    dt = x.dtype
    xp, xs = _rows(x, dt, "x", rows, d, dev)
    dyp, dys = _rows(dy, dt, "dy", rows, d, dev)
    dxp, dxs = (None, d) if dx is None else _rows(dx, dt, "dx", rows, d, dev)
    wsp, wsn = (None, 0) if workspace is None else _workspace(workspace, dev)
    _call(_lib().vp_ln_backward, dev, dyp, dys, xp, xs, _DTYPE_CODE[dt], rows, d, _opt(weight, wdt, "weight", d, dev),
          _DTYPE_CODE[wdt], _ptr(mean, _F32, "mean", rows, dev), _ptr(rstd, _F32, "rstd", rows, dev), dxp, dxs,
          _opt(dweight, wdt, "dweight", d, dev), _opt(dbias, wdt, "dbias", d, dev), wsp, wsn, _stream(stream, dev))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        d = x.shape[-1]
        x2 = x.reshape(-1, d)
        if x2.stride(-1) != 1 or (x2.shape[0] > 1 and x2.stride(0) < d):
            x2 = x2.contiguous()
        weight = None if weight is None else weight.contiguous()
        bias = None if bias is None else bias.contiguous()
        rows = x2.shape[0]
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty(2, rows, dtype=_F32, device=x.device)
        vp_ln_forward(x2, weight, bias, eps, y.view(-1, d) if rows else y.reshape(0, d), stats[0], stats[1])
        ctx.save_for_backward(x2, weight, stats)
        ctx.bias_like = None if bias is None else (bias.shape, bias.dtype)
        ctx.shape = x.shape
        return y

    @staticmethod
    @first_derivative_only
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        rows, d = x.shape
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        dy = dy.reshape(-1, d)
        if dy.stride(-1) != 1 or (rows > 1 and dy.stride(0) < d):       # an expanded or transposed upstream gradient
            dy = dy.contiguous()
        dx = torch.empty(rows, d, dtype=x.dtype, device=x.device) if need_x else None
        dw = torch.empty_like(weight) if need_w and weight is not None else None
        db = torch.empty(ctx.bias_like[0], dtype=ctx.bias_like[1], device=x.device) if need_b and ctx.bias_like else None
        ws = None
        if dw is not None or db is not None:
            ws = torch.empty(vp_ln_workspace_bytes(rows, d), dtype=torch.uint8, device=x.device)
        vp_ln_backward(dy, x, weight, stats[0], stats[1], dx, dw, db, ws)
        return (None if dx is None else dx.view(ctx.shape)), dw, db, None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension, differentiable in x, weight and bias.

    x is bfloat16, float16 or float32 of any shape; weight and bias ``[d]`` have x's dtype or float32 (both the same).
    Statistics are float32; each result is rounded once."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must have a last dimension of at least 1")
    return _LayerNorm.apply(x, weight, bias, float(eps))


# --------------------------------------------------------------------------- post-training losses (sequence_loss.h)
def _packed(logp, mask, seq_offsets):
    dev = _device(logp, "logp")
    T = logp.numel()
    if not isinstance(seq_offsets, torch.Tensor) or seq_offsets.dim() != 1 or seq_offsets.numel() < 1:
        raise ValueError("seq_offsets must be a one-dimensional tensor with one entry more than there are sequences")
    n = seq_offsets.numel() - 1
    mp = None
    if mask is not None:
        mp = _ptr(mask, torch.uint8 if mask.dtype is torch.uint8 else torch.bool, "mask", T, dev)
    return dev, T, n, _ptr(logp, _F32, "logp", T, dev), mp, _ptr(seq_offsets, torch.int64, "seq_offsets", n + 1, dev)


def _choice(table, value, name: str) -> int:
    try:
        return table[value]
    except KeyError:
        raise ValueError(f"{name} must be one of {sorted(table)}, got {value!r}") from None


def vp_policy_loss_workspace_bytes(T: int, n_seqs: int) -> int:
    return _lib().vp_policy_loss_workspace_bytes(T, n_seqs)


def _policy_args(logp, old_logp, ref_logp, advantages, mask, seq_offsets, clip_low, clip_high, kl_coef, aggregate, per_token):
    dev, T, n, lp, mp, op = _packed(logp, mask, seq_offsets)
    if not isinstance(advantages, torch.Tensor) or advantages.numel() not in (T, n):
        raise ValueError(f"advantages must have one entry per token ({T}) or per sequence ({n})")
    if per_token is None:
        per_token = advantages.numel() == T
    return dev, (lp, _ptr(old_logp, _F32, "old_logp", T, dev), _opt(ref_logp, _F32, "ref_logp", T, dev),
                 _ptr(advantages, _F32, "advantages", T if per_token else n, dev), 1 if per_token else 0, mp, op, T, n,
                 clip_low, clip_high, kl_coef, _choice(_AGGREGATE, aggregate, "aggregate")), T


def vp_policy_loss(logp, old_logp, ref_logp, advantages, mask, seq_offsets, clip_low: float, clip_high: float, kl_coef: float,
                   aggregate: str, stats, dlogp, workspace, upstream=None, adv_per_token: Optional[bool] = None,
                   stream=None) -> None:
    """Clipped policy loss with a KL term over packed sequences: stats [4] = loss and the means over valid tokens of the KL
    estimate, of "clipped" and of the ratio; dlogp [T] (None: forward only) = upstream * dloss/dlogp.  aggregate is
    "token_mean" or "seq_mean"; advantages has one entry per token or one per sequence, told apart by their number unless
    adv_per_token says which (per token where both counts are the same); mask is bool or uint8 [T] or None.  See include/sequence_loss.h."""
    dev, args, T = _policy_args(logp, old_logp, ref_logp, advantages, mask, seq_offsets, clip_low, clip_high, kl_coef, aggregate,
                                adv_per_token)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_policy_loss, dev, *args, _ptr(stats, _F32, "stats", 4, dev), _opt(dlogp, _F32, "dlogp", T, dev),
          _opt(upstream, _F32, "upstream", 1, dev), wsp, wsn, _stream(stream, dev))


def vp_policy_loss_backward(logp, old_logp, ref_logp, advantages, mask, seq_offsets, clip_low: float, clip_high: float,
                            kl_coef: float, aggregate: str, dlogp, workspace, upstream=None,
                            adv_per_token: Optional[bool] = None, stream=None) -> None:
    """The gradient alone, after vp_policy_loss with the same inputs, settings and workspace."""
    dev, args, T = _policy_args(logp, old_logp, ref_logp, advantages, mask, seq_offsets, clip_low, clip_high, kl_coef, aggregate,
                                adv_per_token)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_policy_loss_backward, dev, *args, _ptr(dlogp, _F32, "dlogp", T, dev),
          _opt(upstream, _F32, "upstream", 1, dev), wsp, wsn, _stream(stream, dev))


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, old_logp, ref_logp, advantages, mask, seq_offsets, cfg):
        logp = logp.contiguous()
        ws = torch.empty(vp_policy_loss_workspace_bytes(logp.numel(), seq_offsets.numel() - 1), dtype=torch.uint8, device=logp.device)
        stats = torch.empty(4, dtype=_F32, device=logp.device)
        vp_policy_loss(logp, old_logp, ref_logp, advantages, mask, seq_offsets, *cfg[:4], stats, None, ws, adv_per_token=cfg[4])
        ctx.save_for_backward(logp, old_logp, ref_logp, advantages, mask, seq_offsets, ws)
        ctx.cfg = cfg
        ctx.mark_non_differentiable(stats)
        return stats[0].clone(), stats

    @staticmethod
    @first_derivative_only
    def backward(ctx, g, _):
        *inputs, ws = ctx.saved_tensors
        dlogp = torch.empty_like(inputs[0])
        vp_policy_loss_backward(*inputs, *ctx.cfg[:4], dlogp, ws, upstream=g.to(_F32).reshape(1).contiguous(), adv_per_token=ctx.cfg[4])
        return dlogp, None, None, None, None, None, None


def policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, seq_offsets: torch.Tensor,
                mask: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, aggregate: str = "token_mean",
                adv_per_token: Optional[bool] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss, stats) of the clipped policy objective over packed sequences; loss is a scalar, differentiable in logp.

    With the head of this package, ``logp = -vocab_proj_cross_entropy(H, W, labels)``.  Tokens whose mask is false (prompts,
    padding) may hold anything and get no gradient.  stats [4]: loss, mean KL estimate, clipped share, mean ratio.

    The mean is over this call's tokens (or sequences).  Of a batch in parts, over ranks or accumulated, back-propagate
    ``loss * (n / N)`` of each part: n valid tokens here (``mask.sum()``), N in all parts."""
    cfg = (float(clip_low), float(clip_high), float(kl_coef), aggregate, adv_per_token)
    return _PolicyLoss.apply(logp, old_logp, ref_logp, advantages, mask, seq_offsets, cfg)


def vp_preference_loss_workspace_bytes(T: int, n_pairs: int) -> int:
    return _lib().vp_preference_loss_workspace_bytes(T, n_pairs)


def _pairs(n_seqs: int) -> int:
    if n_seqs % 2:
        raise ValueError(f"a preference loss needs an even number of sequences (preferred ones first), got {n_seqs}")
    return n_seqs // 2


def vp_preference_loss(logp, ref_logp, mask, seq_offsets, beta: float, margin: float, label_smoothing: float, kind: str,
                       average: bool, stats, rewards, dlogp, workspace, upstream=None, stream=None) -> None:
    """Preference loss over packed sequences, the preferred answers first and their counterparts in the same order behind
    them: stats [3] = loss, share of pairs won, mean reward gap; rewards [2 pairs] (or None); dlogp [T] (or None) = upstream *
    dloss/dlogp.  kind is "sigmoid" or "ipo"; ref_logp None means zeros.  See include/sequence_loss.h."""
    dev, T, n, lp, mp, op = _packed(logp, mask, seq_offsets)
    pairs = _pairs(n)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_preference_loss, dev, lp, _opt(ref_logp, _F32, "ref_logp", T, dev), mp, op, T, pairs, beta, margin,
          label_smoothing, _choice(_KIND, kind, "kind"), 1 if average else 0, _ptr(stats, _F32, "stats", 3, dev),
          _opt(rewards, _F32, "rewards", n, dev), _opt(dlogp, _F32, "dlogp", T, dev), _opt(upstream, _F32, "upstream", 1, dev),
          wsp, wsn, _stream(stream, dev))


def vp_preference_loss_backward(mask, seq_offsets, dlogp, workspace, upstream=None, stream=None) -> None:
    """The gradient alone, after vp_preference_loss with the same inputs, settings and workspace."""
    dev, T, n, dp, mp, op = _packed(dlogp, mask, seq_offsets)
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().vp_preference_loss_backward, dev, mp, op, T, _pairs(n), dp, _opt(upstream, _F32, "upstream", 1, dev), wsp, wsn,
          _stream(stream, dev))


class _PreferenceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, ref_logp, mask, seq_offsets, cfg):
        logp = logp.contiguous()
        n = seq_offsets.numel() - 1
        ws = torch.empty(vp_preference_loss_workspace_bytes(logp.numel(), n // 2), dtype=torch.uint8, device=logp.device)
        stats = torch.empty(3, dtype=_F32, device=logp.device)
        rewards = torch.empty(n, dtype=_F32, device=logp.device)
        vp_preference_loss(logp, ref_logp, mask, seq_offsets, *cfg, stats, rewards, None, ws)
        ctx.save_for_backward(mask, seq_offsets, ws)
        ctx.like = (logp.shape, logp.device)
        ctx.mark_non_differentiable(stats, rewards)
        return stats[0].clone(), stats, rewards

    @staticmethod
    @first_derivative_only
    def backward(ctx, g, _stats, _rewards):
        mask, seq_offsets, ws = ctx.saved_tensors
        dlogp = torch.empty(ctx.like[0], dtype=_F32, device=ctx.like[1])
        vp_preference_loss_backward(mask, seq_offsets, dlogp, ws, upstream=g.to(_F32).reshape(1).contiguous())
        return dlogp, None, None, None, None


def preference_loss(logp: torch.Tensor, seq_offsets: torch.Tensor, ref_logp: Optional[torch.Tensor] = None,
                    mask: Optional[torch.Tensor] = None, beta: float = 0.1, margin: float = 0.0, label_smoothing: float = 0.0,
                    kind: str = "sigmoid", average: bool = False) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(loss, stats, rewards) of a preference objective over packed sequences; loss is a scalar, differentiable in logp.

    The first half of the sequences are the preferred answers, the second half their counterparts in the same order.
    stats [3]: loss, share of pairs won, mean reward gap; rewards [sequences]: beta times the (mean) log ratio."""
    cfg = (float(beta), float(margin), float(label_smoothing), kind, bool(average))
    return _PreferenceLoss.apply(logp, ref_logp, mask, seq_offsets, cfg)


# --------------------------------------------------------------------------- Muon (muon.h)
def muon_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return _lib().muon_workspace_bytes(batch, rows, cols)


def muon_rms_scale(rows: int, cols: int) -> float:
    """The `scale` that gives an orthogonalised update about AdamW's root mean square (0.2), whatever the shape."""
    return 0.2 * math.sqrt(max(rows, cols))


def _matrices(t, name: str) -> Tuple[int, int, int]:
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be [rows, cols] or [batch, rows, cols], got {list(t.shape)}")
    return (1 if t.dim() == 2 else t.shape[0]), t.shape[-2], t.shape[-1]


def _float_code(t, name: str) -> int:
    if t.dtype not in _DTYPE_CODE:
        raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
    return _DTYPE_CODE[t.dtype]


def _coeffs(coeffs, steps: int):
    """None, one (a, b, c) for every step, or one triple per step -> HOST double [steps][3]."""
    if coeffs is None:
        return None
    flat = [float(v) for v in coeffs] if not isinstance(coeffs[0], Sequence) else [float(v) for c in coeffs for v in c]
    if len(flat) == 3:
        flat = flat * steps
    if len(flat) != 3 * steps:
        raise ValueError(f"coeffs must be one triple or {steps} triples")
    return (ctypes.c_double * len(flat))(*flat)


def muon_orthogonalize(G, O, workspace, coeffs=None, steps: int = 5, eps: float = 1e-7, stream=None) -> None:
    """O = G orthogonalised by `steps` Newton-Schulz steps, for one matrix [rows, cols] or a batch of them.  O has G's shape
    and may have another float type, or be G itself.  See include/muon.h."""
    dev = _device(G, "G")
    batch, rows, cols = _matrices(G, "G")
    n = batch * rows * cols
    gc, oc = _float_code(G, "G"), _float_code(O, "O")
    if O.shape != G.shape:
        raise ValueError(f"O must have G's shape {list(G.shape)}, got {list(O.shape)}")
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().muon_orthogonalize, dev, _ptr(G, G.dtype, "G", n, dev), gc, _ptr(O, O.dtype, "O", n, dev), oc, batch, rows, cols,
          _coeffs(coeffs, steps), steps, eps, wsp, wsn, _stream(stream, dev))


def muon_step(p, m, grad, w_bf16, lr: float, mu: float, weight_decay: float, scale: float, workspace, nesterov: bool = True,
              coeffs=None, steps: int = 5, eps: float = 1e-7, stream=None) -> None:
    """One Muon update of one matrix [rows, cols] or a batch of one shape: p (float32 master) and m (float32 momentum) in
    place, w_bf16 (working weight, may be None) written.  `scale` multiplies the orthogonalised update; muon_rms_scale gives
    AdamW's update size.  See include/muon.h."""
    dev = _device(p, "p")
    batch, rows, cols = _matrices(p, "p")
    n = batch * rows * cols
    gc = _float_code(grad, "grad") if isinstance(grad, torch.Tensor) else 2
    for t, name in ((m, "m"), (grad, "grad"), (w_bf16, "w_bf16")):
        if isinstance(t, torch.Tensor) and t.shape != p.shape:
            raise ValueError(f"{name} must have p's shape {list(p.shape)}, got {list(t.shape)}")
    wsp, wsn = _workspace(workspace, dev)
    _call(_lib().muon_step, dev, _ptr(p, _F32, "p", n, dev), _ptr(m, _F32, "m", n, dev),
          _ptr(grad, getattr(grad, "dtype", None), "grad", n, dev), gc, _opt(w_bf16, _BF16, "w_bf16", n, dev), batch, rows, cols, lr, mu,
          1 if nesterov else 0, weight_decay, scale, _coeffs(coeffs, steps), steps, eps, wsp, wsn, _stream(stream, dev))


def muon_device_status(workspace, stream=None) -> int:
    """The status word of the last call that used this workspace (synchronises): 0, or 2 when a wait ran out."""
    dev = _device(workspace, "workspace")
    out = ctypes.c_int32(-1)
    _call(_lib().muon_device_status, dev, _workspace(workspace, dev)[0], ctypes.byref(out), _stream(stream, dev))
    return int(out.value)


def muon_debug_drop(kernel_kind: int, index: int = 0, cta_ranks: int = 1) -> None:
    """Test hook: a signal of the next Muon launch of that kind gets lost (see include/muon.h); kernel_kind < 0 disarms."""
    code = _lib().muon_debug_drop(kernel_kind, index, cta_ranks)
    if code:
        _fail(code)
