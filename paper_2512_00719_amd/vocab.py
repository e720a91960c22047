"""The operators at a model's vocabulary (``include/simple_vocab.h``) over torch device tensors.

A decoding step is ``embed`` -> the model -> ``rms_norm_int8`` -> ``linear_int8`` -> a sampling call of
``binding``; a training step ends with ``rms_norm`` -> ``linear_xent`` and begins its backward pass with
``linear_xent_grad`` -> ``rms_norm_grad`` ... ``embed_grad``.  As in ``binding`` only arguments are checked and marshalled here:
every step runs in the HIP kernels of the library, on the current stream, without a synchronisation.  Outputs and workspaces are allocated by torch
where they are not passed.

Automatic differentiation records none of these calls: gradients are calls of their own.  A tensor that requires a gradient is refused (``ValueError``) unless gradients
are off (``torch.no_grad()``), so that a loss does not silently lose a term; a tensor that is passed for an output counts as modified in place.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding
from .binding import SIMPLE_BF16, SIMPLE_F32, SIMPLE_OK, SimpleError, _addresses, _current_stream

EXPORTS = ("simple_rms_norm", "simple_rms_norm_int8", "simple_quantize_rows", "simple_rms_norm_grad", "simple_rms_norm_grad_workspace",
           "simple_embed", "simple_embed_grad", "simple_embed_grad_workspace", "simple_linear_int8", "simple_linear_int8_workspace",
           "simple_xent", "simple_xent_workspace", "simple_xent_workspace_aligned", "simple_xent_grad", "simple_xent_grad_workspace",
           "simple_xent_grad_workspace_aligned")


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    vp, i64, f32, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_int
    signatures = {
        "simple_rms_norm": (ci, vp, i64, vp, i64, vp, i64, i64, ci, f32, vp, i64, vp, i64, vp, vp),
        "simple_rms_norm_int8": (ci, vp, i64, vp, i64, vp, i64, i64, ci, f32, vp, i64, vp, i64, vp, vp),
        "simple_quantize_rows": (ci, vp, i64, i64, i64, ci, vp, i64, vp, vp),
        "simple_rms_norm_grad": (ci, vp, i64, vp, i64, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp, vp, i64, vp),
        "simple_rms_norm_grad_workspace": (i64, i64, i64),
        "simple_embed": (ci, vp, vp, i64, i64, i64, i64, ci, f32, vp, i64, vp),
        "simple_embed_grad": (ci, vp, vp, i64, i64, i64, i64, ci, f32, vp, i64, ci, ci, vp, i64, vp),
        "simple_embed_grad_workspace": (i64, i64, i64, i64),
        "simple_linear_int8": (ci, vp, i64, vp, vp, i64, vp, i64, i64, i64, vp, i64, ci, vp, i64, vp),
        "simple_linear_int8_workspace": (i64, i64, i64, i64),
        "simple_xent": (ci, vp, i64, vp, i64, vp, i64, i64, i64, f32, vp, vp, vp, i64, vp),
        "simple_xent_workspace": (i64, i64, i64, i64),
        "simple_xent_workspace_aligned": (i64, i64, i64, i64),
        "simple_xent_grad": (ci, vp, vp, i64, vp, i64, vp, vp, i64, i64, i64, f32, vp, i64, vp, i64, ci, ci, vp, i64, vp),
        "simple_xent_grad_workspace": (i64, i64, i64, i64, ci, ci),
        "simple_xent_grad_workspace_aligned": (i64, i64, i64, i64, ci, ci),
    }
    assert set(signatures) == set(EXPORTS)
    for name, (restype, *argtypes) in signatures.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = restype, argtypes
    return lib


_lib = _declare(binding._lib)
_TYPES = {torch.float32: SIMPLE_F32, torch.bfloat16: SIMPLE_BF16}


def _check(rc: int, where: str) -> None:
    if rc != SIMPLE_OK:
        raise SimpleError(rc, where)


def _dtype(t: torch.Tensor, name: str) -> int:
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise TypeError(f"{name} is float32 or bfloat16, got {t.dtype}") from None


def _refuse_recording(name: str) -> None:
    if torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this call does not record: pass it detached, or call under torch.no_grad()")


# (These run ahead of every call, whose kernels may take 5 us: the usual case is one expression.)
def _tensor(t: torch.Tensor, name: str, shape, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    """`t`, if it is a tensor of that kind on that device whose rows are dense (the last dimension's stride is 1)."""
    if t.requires_grad:
        _refuse_recording(name)
    if t.dtype is dtype and t.shape == shape and t.device == device and (t.is_contiguous() or t.stride(-1) == 1 or t.shape[-1] == 1):
        return t
    if t.dtype is not dtype:
        raise TypeError(f"{name} is {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, others on {device}")
    raise ValueError(f"{name} has a stride of {t.stride(-1)} along its rows: 1 is wanted")


def _matrix(t: torch.Tensor, name: str, dtypes=(torch.float32, torch.bfloat16)) -> torch.device:
    """The device of a [rows, values] matrix on the current GPU, the first operand of a call."""
    if t.dim() != 2 or t.shape[1] == 0:
        raise ValueError(f"{name} is [rows, values], got shape {tuple(t.shape)}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} is one of {dtypes}, got {t.dtype}")
    if t.requires_grad:
        _refuse_recording(name)
    device = t.device
    if device.type != "cuda" or device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {device}: the current GPU is wanted")
    if not t.is_contiguous():
        _tensor(t, name, t.shape, t.dtype, device)
    return device


def _stride(t: Optional[torch.Tensor]) -> int:
    """Row stride in elements.  (torch says anything for a single row.)"""
    if t is None:
        return 0
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _out(t: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _tensor(t, name, shape, dtype, device)
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)
    return t


def _workspace(nbytes: int, where: str, device: torch.device) -> torch.Tensor:
    if nbytes < 0:
        raise SimpleError(nbytes, where)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _norm_inputs(x, weight, residual, h):
    _matrix(x, "x")
    _tensor(weight, "weight", (x.shape[1],), x.dtype, x.device)
    if residual is None:
        if h is not None:
            raise ValueError("h is the sum with a residual, and there is none")
        return None
    _tensor(residual, "residual", x.shape, x.dtype, x.device)
    return _out(h, "h", x.shape, x.dtype, x.device)


def rms_norm(x, weight, *, eps: float = 1e-6, residual=None, h=None, out=None, rstd=None, need_rstd: bool = False):
    """``(y, h, rstd)``: h = x + residual (x itself without one), y = h / rms(h) * weight in x's type, rstd = 1 / rms(h) (float32 [T],
    ``None`` unless ``need_rstd`` or a tensor for it is given).  ``h`` may be ``residual``, ``out`` may be ``x``."""
    total = _norm_inputs(x, weight, residual, h)
    T, D = x.shape
    out = _out(out, "out", x.shape, x.dtype, x.device)
    if rstd is not None or need_rstd:
        rstd = _out(rstd, "rstd", (T,), torch.float32, x.device)
    _check(_lib.simple_rms_norm(x.data_ptr(), _stride(x), _ptr(residual), _stride(residual), weight.data_ptr(), T, D, _TYPES[x.dtype], eps,
                                _ptr(total), _stride(total), out.data_ptr(), _stride(out), _ptr(rstd), _current_stream()), "simple_rms_norm")
    return out, x if total is None else total, rstd


def rms_norm_int8(x, weight, *, eps: float = 1e-6, residual=None, h=None, codes=None, scales=None):
    """``(codes, scales, h)``: the norm's output as int8 [T, D] and float32 [T], code * scale."""
    total = _norm_inputs(x, weight, residual, h)
    T, D = x.shape
    codes = _out(codes, "codes", x.shape, torch.int8, x.device)
    scales = _out(scales, "scales", (T,), torch.float32, x.device)
    _check(_lib.simple_rms_norm_int8(x.data_ptr(), _stride(x), _ptr(residual), _stride(residual), weight.data_ptr(), T, D, _TYPES[x.dtype], eps,
                                     _ptr(total), _stride(total), codes.data_ptr(), _stride(codes), scales.data_ptr(), _current_stream()),
           "simple_rms_norm_int8")
    return codes, scales, x if total is None else total


def quantize_rows(x, *, codes=None, scales=None):
    """``(codes, scales)``: rows as int8 and float32 [T], code * scale.  For the weights of ``linear_int8``, once."""
    _matrix(x, "x")
    T, D = x.shape
    codes = _out(codes, "codes", x.shape, torch.int8, x.device)
    scales = _out(scales, "scales", (T,), torch.float32, x.device)
    _check(_lib.simple_quantize_rows(x.data_ptr(), _stride(x), T, D, _TYPES[x.dtype], codes.data_ptr(), _stride(codes), scales.data_ptr(),
                                     _current_stream()), "simple_quantize_rows")
    return codes, scales


def rms_norm_grad(dy, h, weight, rstd, *, dh=None, dx=None, dweight=None):
    """``(dx, dweight)``: gradients of ``rms_norm`` for x (and residual alike; ``dh`` is what reaches h past the norm) and for its weight
    (float32 [D]).  ``dx`` may be ``dy`` or ``dh``."""
    _matrix(dy, "dy")
    T, D = dy.shape
    _tensor(h, "h", dy.shape, dy.dtype, dy.device)
    _tensor(weight, "weight", (D,), dy.dtype, dy.device)
    _tensor(rstd, "rstd", (T,), torch.float32, dy.device)
    if dh is not None:
        _tensor(dh, "dh", dy.shape, dy.dtype, dy.device)
    dx = _out(dx, "dx", dy.shape, dy.dtype, dy.device)
    dweight = _out(dweight, "dweight", (D,), torch.float32, dy.device)
    ws = _workspace(_lib.simple_rms_norm_grad_workspace(T, D), "simple_rms_norm_grad_workspace", dy.device)
    _check(_lib.simple_rms_norm_grad(dy.data_ptr(), _stride(dy), h.data_ptr(), _stride(h), weight.data_ptr(), rstd.data_ptr(), _ptr(dh),
                                     _stride(dh), T, D, _TYPES[dy.dtype], dx.data_ptr(), _stride(dx), dweight.data_ptr(), ws.data_ptr(),
                                     ws.numel(), _current_stream()), "simple_rms_norm_grad")
    return dx, dweight


def embed(ids, table, *, scale: float = 1.0, out=None):
    """Rows ``ids`` (int32 [T]) of ``table`` [V, D], times ``scale``.  An id outside the vocabulary gives a row of zeros."""
    _matrix(table, "table")
    V, D = table.shape
    T = ids.numel()
    _tensor(ids, "ids", (T,), torch.int32, table.device)
    out = _out(out, "out", (T, D), table.dtype, table.device)
    _check(_lib.simple_embed(ids.data_ptr(), table.data_ptr(), _stride(table), T, V, D, _TYPES[table.dtype], scale, out.data_ptr(), _stride(out),
                             _current_stream()), "simple_embed")
    return out


def embed_grad(ids, dout, V: int, *, scale: float = 1.0, dtable=None, accumulate: bool = False):
    """Gradient of ``embed`` for its table, [V, D] in dout's type, or in that of ``dtable`` (float32 or bfloat16) where it is given;
    ``accumulate`` adds it to what ``dtable`` holds."""
    _matrix(dout, "dout")
    T, D = dout.shape
    _tensor(ids, "ids", (T,), torch.int32, dout.device)
    if dtable is None:
        if accumulate:
            raise ValueError("accumulate adds to dtable, and there is none")
        dtable = torch.empty((V, D), dtype=dout.dtype, device=dout.device)
    else:
        _dtype(dtable, "dtable")
        _out(dtable, "dtable", (V, D), dtable.dtype, dout.device)
    ws = _workspace(_lib.simple_embed_grad_workspace(T, V, D), "simple_embed_grad_workspace", dout.device)
    _check(_lib.simple_embed_grad(ids.data_ptr(), dout.data_ptr(), _stride(dout), T, V, D, _TYPES[dout.dtype], scale, dtable.data_ptr(),
                                  _stride(dtable), _TYPES[dtable.dtype], int(accumulate), ws.data_ptr(), ws.numel(), _current_stream()),
           "simple_embed_grad")
    return dtable


def linear_int8(codes, scales, w_codes, w_scales, *, out_dtype: torch.dtype = torch.float32, out=None):
    """Logits [T, V] of ``out_dtype`` (float32 or bfloat16): codes [T, K] times w_codes [V, K], both int8, times scales [T] and w_scales [V]."""
    _matrix(codes, "codes", (torch.int8,))
    T, K = codes.shape
    V = w_codes.shape[0]
    _tensor(scales, "scales", (T,), torch.float32, codes.device)
    _tensor(w_codes, "w_codes", (V, K), torch.int8, codes.device)
    _tensor(w_scales, "w_scales", (V,), torch.float32, codes.device)
    if out is not None:
        out_dtype = out.dtype
    if out_dtype not in _TYPES:
        raise TypeError(f"logits are float32 or bfloat16, got {out_dtype}")
    out = _out(out, "out", (T, V), out_dtype, codes.device)
    ws = None
    if (codes.data_ptr() | w_codes.data_ptr() | _stride(codes) | _stride(w_codes) | K) % 16:  # rows that are not aligned
        ws = _workspace(_lib.simple_linear_int8_workspace(T, V, K), "simple_linear_int8_workspace", codes.device)
    _check(_lib.simple_linear_int8(codes.data_ptr(), _stride(codes), scales.data_ptr(), w_codes.data_ptr(), _stride(w_codes), w_scales.data_ptr(),
                                   T, V, K, out.data_ptr(), _stride(out), _TYPES[out_dtype], _ptr(ws), 0 if ws is None else ws.numel(),
                                   _current_stream()), "simple_linear_int8")
    return out


def _xent_inputs(hidden, weight, targets):
    _matrix(hidden, "hidden", (torch.bfloat16,))
    T, D = hidden.shape
    V = weight.shape[0]
    _tensor(weight, "weight", (V, D), torch.bfloat16, hidden.device)
    _tensor(targets, "targets", (T,), torch.int32, hidden.device)
    return T, V, D


def _aligned(hidden, weight) -> bool:
    """Whether the rows of both start at multiples of 16 bytes and are as long, so that a call has no copies of them."""
    h, w = _stride(hidden), _stride(weight)
    return (hidden.data_ptr() | weight.data_ptr()) % 16 == 0 and (h | w | hidden.shape[1]) % 8 == 0 and max(h, w) <= 1 << 21


def linear_xent(hidden, weight, targets, *, logit_scale: float = 1.0, loss=None, lse=None):
    """``(loss, lse)``, float32 [T]: negative log-probability of ``targets`` (int32; outside the vocabulary: 0) under the logits
    ``logit_scale * hidden @ weight.T``, and the logarithm of the sum of their exponentials.  bfloat16 operands."""
    T, V, D = _xent_inputs(hidden, weight, targets)
    loss = _out(loss, "loss", (T,), torch.float32, hidden.device)
    lse = _out(lse, "lse", (T,), torch.float32, hidden.device)
    size = _lib.simple_xent_workspace_aligned if _aligned(hidden, weight) else _lib.simple_xent_workspace
    ws = _workspace(size(T, V, D), "simple_xent_workspace", hidden.device)
    _check(_lib.simple_xent(hidden.data_ptr(), _stride(hidden), weight.data_ptr(), _stride(weight), targets.data_ptr(), T, V, D, logit_scale,
                            loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), _current_stream()), "simple_xent")
    return loss, lse


def linear_xent_grad(dloss, hidden, weight, targets, lse, *, logit_scale: float = 1.0, dhidden=None, dweight=None, accumulate: bool = False,
                     need_dhidden: bool = True, need_dweight: bool = True):
    """``(dhidden, dweight)``: gradients of ``(dloss * linear_xent(...)[0]).sum()``, in bfloat16 (``dweight`` in the type of the tensor given for it,
    bfloat16 or float32, to which ``accumulate`` adds).  What is not needed is not formed and ``None``.  Of more than 64 tokens the logits' gradient has 11 bits
    within 2^-28 of a token's largest element, and fewer below (``include/simple_vocab.h``)."""
    T, V, D = _xent_inputs(hidden, weight, targets)
    _tensor(dloss, "dloss", (T,), torch.float32, hidden.device)
    _tensor(lse, "lse", (T,), torch.float32, hidden.device)
    dhidden = _out(dhidden, "dhidden", (T, D), torch.bfloat16, hidden.device) if need_dhidden else None
    if accumulate and need_dweight and dweight is None:
        raise ValueError("accumulate adds to dweight, and there is none")
    if not need_dweight:
        dweight = None
    elif dweight is None:
        dweight = torch.empty((V, D), dtype=torch.bfloat16, device=hidden.device)
    else:
        _dtype(dweight, "dweight")
        _out(dweight, "dweight", (V, D), dweight.dtype, hidden.device)
    size = _lib.simple_xent_grad_workspace_aligned if _aligned(hidden, weight) else _lib.simple_xent_grad_workspace
    ws = _workspace(size(T, V, D, int(need_dhidden), int(need_dweight)), "simple_xent_grad_workspace", hidden.device)
    _check(_lib.simple_xent_grad(dloss.data_ptr(), hidden.data_ptr(), _stride(hidden), weight.data_ptr(), _stride(weight), targets.data_ptr(),
                                 lse.data_ptr(), T, V, D, logit_scale, _ptr(dhidden), _stride(dhidden), _ptr(dweight), _stride(dweight),
                                 SIMPLE_BF16 if dweight is None else _TYPES[dweight.dtype], int(accumulate), ws.data_ptr(), ws.numel(),
                                 _current_stream()), "simple_xent_grad")
    return dhidden, dweight
