"""Layer norms in front of a projection, with a weight and a bias or modulated by a scale and a shift for each batch, forward
and backward.

    scale, shift = modulation.chunk(6, dim=-1)[:2]            # of adaln_int4_linear's output, [batch, 6 N]
    y = layer_norm_modulate(x, scale, shift)                  # x [batch, token, N] -> what rpbh_quantize_act takes
    dx, dscale, dshift = layer_norm_modulate_backward(dy, x, scale)

Rows are tensors [batch, token, N] or [token, N] of bf16 or fp32 values whose last dimension is contiguous.
"""

import ctypes
import struct

import torch

from . import ORBIT_OUT_BF16, ORBIT_OUT_F32, _call, _check, _ptr, lib
from .attention_input import _rows_apart

_TYPES = {torch.float32: ORBIT_OUT_F32, torch.bfloat16: ORBIT_OUT_BF16}

_pack_rows = struct.Struct("Pqqi4x").pack   # orbit_rows as bytes: data, strides of batch and row, dtype


def _rows(t, name, like=None, dtype=None):
    """(t's rows for the library, its [batch, token, N]).  `like`: the tensor whose shape and device it must have."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU")
    kind = _TYPES.get(t.dtype)
    if kind is None or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'bf16 or fp32'}, got {t.dtype}")
    shape = t.shape
    if like is not None and (shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must have the shape {tuple(like.shape)} on {like.device}, got {tuple(shape)} on {t.device}")
    if len(shape) == 3:
        sb, sl, sn = t.stride()
    elif len(shape) == 2:
        sl, sn = t.stride()
        sb, shape = 0, (1, *shape)
    else:
        raise ValueError(f"{name} must be [batch, token, N] or [token, N]")
    if sn != 1 and shape[2] > 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return _pack_rows(t.data_ptr(), sb, sl, kind), shape


# A single token's norm takes 3.5 us on the device and the host's part of a call twice that, so it is kept short: 8.7 -> 8.0 us.
def _output(out, like, name, dtype):
    """(out, its rows): the caller's output, checked, or a new one of `like`'s shape."""
    if out is None:
        out = torch.empty_like(like, dtype=dtype)      # in like's order of dimensions, for sliding windows in another one
        if out.stride(-1) != 1:
            out = torch.empty(like.shape, dtype=dtype, device=like.device)
        return out, _pack_rows(out.data_ptr(), out.stride(0) if out.dim() == 3 else 0, out.stride(-2), _TYPES[dtype])
    rows = _rows(out, name, like, dtype)[0]
    _rows_apart(out, name)
    return out, rows


def _weight(w, name, shape, dev):
    """(pointer, batch stride) of a weight [N], or [B, N] with contiguous rows."""
    if w is None:
        return None, 0
    if not isinstance(w, torch.Tensor) or w.dtype not in _TYPES:
        raise ValueError(f"{name} must be a bf16 or fp32 tensor")
    if w.shape != shape or w.device != dev or (w.stride(-1) != 1 and shape[-1] > 1):
        raise ValueError(f"{name} must have the shape {tuple(shape)} and contiguous rows on {dev}, got {tuple(w.shape)} on {w.device}")
    return w.data_ptr(), w.stride(0) if len(shape) == 2 else 0


def _forward(x, weight, bias, names, modulate, eps, out_dtype, out):
    hx, (B, L, N) = _rows(x, "x")
    if out_dtype is None:
        out_dtype = x.dtype if out is None else out.dtype
    if out_dtype not in _TYPES:
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    shape, dev = (B, N) if modulate else (N,), x.device
    w, w_batch = _weight(weight, names[0], shape, dev)
    b, b_batch = _weight(bias, names[1], shape, dev)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError(f"{names[0]} and {names[1]} must be of one type")
    w_dtype = _TYPES[weight.dtype] if weight is not None else _TYPES[bias.dtype] if bias is not None else ORBIT_OUT_F32
    out, hy = _output(out, x, "out", out_dtype)
    _call("layer_norm", dev, hx, hy, B, L, N, w, w_batch, b, b_batch, w_dtype, modulate, eps)
    return out


_workspace_bytes = {}


def _workspace(B, L, N, per_batch, dev):
    """A workspace and its bytes, which the sizes and the device alone decide."""
    key = (B, L, N, per_batch, dev)
    n = _workspace_bytes.get(key)      # read once: another thread may empty the list
    if n is None:
        size = ctypes.c_size_t(0)
        with torch.cuda.device(dev):
            _check("layer_norm_backward_workspace_size", lib().layer_norm_backward_workspace_size(B, L, N, per_batch, ctypes.byref(size)))
        if len(_workspace_bytes) > 1024:
            _workspace_bytes.clear()
        n = _workspace_bytes[key] = size.value
    return torch.empty((max(n, 16),), dtype=torch.uint8, device=dev), n


def _backward(dy, x, weight, name, modulate, eps, x_grad):
    hx, (B, L, N) = _rows(x, "x")
    hdy, _ = _rows(dy, "dy", x)
    w, w_batch = _weight(weight, name, (B, N) if modulate else (N,), x.device)
    w_dtype = ORBIT_OUT_F32 if weight is None else _TYPES[weight.dtype]
    x_grad, hdx = _output(x_grad, x, "x_grad", x.dtype)
    dw, db = (torch.empty((B, N) if modulate else (N,), dtype=torch.float32, device=x.device) for _ in range(2))
    ws, ws_bytes = _workspace(B, L, N, modulate, x.device)
    _call("layer_norm_backward", x.device, hdy, hx, hdx, B, L, N, w, w_batch, w_dtype, modulate, eps, dw.data_ptr(), db.data_ptr(),
          modulate, _ptr(ws), ws_bytes)
    return x_grad, dw, db


def layer_norm(x: torch.Tensor, weight: torch.Tensor = None, bias: torch.Tensor = None, eps: float = 1e-6,
               out_dtype: torch.dtype = None, out: torch.Tensor = None) -> torch.Tensor:
    """(x - mean) / sqrt(variance + eps) * weight + bias over rows of N values; weight and bias [N], of one type, or None.
    `out` may be x."""
    return _forward(x, weight, bias, ("weight", "bias"), 0, eps, out_dtype, out)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor = None, eps: float = 1e-6, x_grad: torch.Tensor = None):
    """(x_grad in x's type, weight_grad fp32 [N], bias_grad fp32 [N]) from the gradient dy of layer_norm's output and its
    inputs.  `x_grad` may be dy where the types are equal, or x."""
    return _backward(dy, x, weight, "weight", 0, eps, x_grad)


def layer_norm_modulate(x: torch.Tensor, scale: torch.Tensor, shift: torch.Tensor, eps: float = 1e-6, out_dtype: torch.dtype = None,
                        out: torch.Tensor = None) -> torch.Tensor:
    """(x - mean) / sqrt(variance + eps) * (1 + scale) + shift, scale and shift [batch, N] with rows that may lie apart (views
    of the modulation projection's output), or None; x [token, N] is one batch.  `out` may be x."""
    return _forward(x, scale, shift, ("scale", "shift"), 1, eps, out_dtype, out)


def layer_norm_modulate_backward(dy: torch.Tensor, x: torch.Tensor, scale: torch.Tensor, eps: float = 1e-6,
                                 x_grad: torch.Tensor = None):
    """(x_grad in x's type, scale_grad fp32 [batch, N], shift_grad fp32 [batch, N]), as layer_norm_backward."""
    return _backward(dy, x, scale, "scale", 1, eps, x_grad)
