"""Queries and keys between the QKV projection and attention: rotary positions with several axes, and the RMS norm
of each head with that rotation in the same pass, forward and backward.

    plan = rope_plan((44, 42, 42), (21, 30, 52))               # time, height, width: 128 values of a head
    q, k = qk_norm_rope(plan, q, k, positions, q_weight, k_weight)

Heads are tensors [batch, token, head, D] or [token, head, D] of bf16 or fp32 values whose last dimension is
contiguous: views of the projection's output and of attention layouts are taken as they lie.
"""

import ctypes
import struct

import numpy as np
import torch

from . import ORBIT_OUT_BF16, ORBIT_OUT_F32, _c_void_p, _call, _check, _expect, _ptr, lib

_TYPES = {torch.float32: ORBIT_OUT_F32, torch.bfloat16: ORBIT_OUT_BF16}


# orbit_heads as bytes: data, strides of batch, token and head, heads, dtype.  A call on a single token takes a few
# microseconds on the device, so the host's part is kept short here too (a ctypes structure costs three times this).
_pack_heads = struct.Struct("Pqqqii").pack


class RopePlan:
    """Handle of the angles of rotary positions."""

    def __init__(self, handle, dims, lengths, halves):
        self._h, self._destroy = handle, lib().rope_plan_destroy
        self.dims, self.lengths, self.halves = dims, lengths, halves

    @property
    def handle(self):
        return self._h

    def upload(self, device=None):
        """Copies the tables to `device` (default: the current one), as Plan.upload."""
        with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
            _check("rope_plan_upload", lib().rope_plan_upload(self._h))
        return self

    def __del__(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None


def _axes(dims, lengths):
    dims, lengths = tuple(int(d) for d in dims), tuple(int(n) for n in lengths)
    if len(dims) != len(lengths):
        raise ValueError(f"{len(dims)} axes have dims and {len(lengths)} have lengths")
    if any(not 0 <= v < 1 << 31 for v in dims + lengths):
        raise ValueError("dims and lengths must be 32-bit numbers, at least 0")
    return dims, lengths, np.array(dims, dtype=np.int32), np.array(lengths, dtype=np.int32)


def rope_plan(dims, lengths, theta: float = 10000.0, halves: bool = False) -> RopePlan:
    """Angles position * theta^(-2 j / dims[a]) of axes that turn dims[a] values of a head each and have
    lengths[a] positions.  Pairs are neighbours (2p, 2p + 1), or (p, p + sum(dims) / 2) with `halves`."""
    dims, lengths, d, n = _axes(dims, lengths)
    out = _c_void_p()
    _check("rope_plan", lib().rope_plan(len(dims), d.ctypes.data, n.ctypes.data, float(theta), int(bool(halves)), ctypes.byref(out)))
    return RopePlan(out, dims, lengths, bool(halves))


def rope_plan_from_angles(angles, halves: bool = False) -> RopePlan:
    """The same handle from the angles themselves: per axis an array [positions, pairs] (scaled, interpolated or
    learned positions)."""
    angles = [np.ascontiguousarray(a, dtype=np.float64) for a in angles]
    if not angles or any(a.ndim != 2 for a in angles):
        raise ValueError("angles must be an array [positions, pairs] for each axis")
    dims, lengths, d, n = _axes([2 * a.shape[1] for a in angles], [a.shape[0] for a in angles])
    flat = np.concatenate([a.ravel() for a in angles])
    out = _c_void_p()
    _check("rope_plan_from_angles", lib().rope_plan_from_angles(len(dims), d.ctypes.data, n.ctypes.data, flat.ctypes.data,
                                                                int(bool(halves)), ctypes.byref(out)))
    return RopePlan(out, dims, lengths, bool(halves))


def _heads(t, name, like=None, dtype=None):
    """(t's rows for the library, its [batch, token, head, D]).  `like`: the shape it must have, on `like`'s device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU")
    kind = _TYPES.get(t.dtype)
    if kind is None or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'bf16 or fp32'}, got {t.dtype}")
    shape = t.shape
    if like is not None and (shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must have the shape {tuple(like.shape)} on {like.device}, got {tuple(shape)} on {t.device}")
    if len(shape) == 4:
        sb, sl, sh, sd = t.stride()
    elif len(shape) == 3:
        sl, sh, sd = t.stride()
        sb, shape = 0, (1, *shape)
    else:
        raise ValueError(f"{name} must be [batch, token, head, D] or [token, head, D]")
    if sd != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return _pack_heads(t.data_ptr(), sb, sl, sh, shape[2], kind), shape


def _rows_apart(t, name):
    """Refuses an output whose rows share memory."""
    reach = 0
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size > 1:
            if stride <= reach:
                raise ValueError(f"{name}'s rows overlap")
            reach += stride * (size - 1)


def _output(out, like, name, dtype):
    """(out, its rows): the caller's output, checked, or a new one of `like`'s shape."""
    if out is None:
        out = torch.empty(like.shape, dtype=dtype, device=like.device)
        L, H, D = like.shape[-3:]
        return out, _pack_heads(out.data_ptr(), L * H * D, H * D, D, H, _TYPES[dtype])
    rows = _heads(out, name, like, dtype)[0]
    _rows_apart(out, name)
    return out, rows


def _positions(plan, positions, B, L, dev):
    """(pointer, elements from one batch's positions to the next's)."""
    if plan is None:
        if positions is not None:
            raise ValueError("positions are given without a plan")
        return None, 0
    if not isinstance(plan, RopePlan):
        raise ValueError("plan must be a RopePlan")
    A = len(plan.dims)
    if not isinstance(positions, torch.Tensor):
        raise ValueError("positions must be a tensor")
    _expect(positions, "positions", torch.int32, (B, L, A) if positions.dim() == 3 else (L, A), dev)
    return positions.data_ptr(), L * A if positions.dim() == 3 else 0


def axial_rope(plan: RopePlan, x: torch.Tensor, positions: torch.Tensor, inverse: bool = False,
               out: torch.Tensor = None) -> torch.Tensor:
    """x's heads turned by the angles of their tokens' positions, int32 [token, axis] or [batch, token, axis];
    `inverse` turns back, which is the gradient: dx = axial_rope(plan, dy, positions, inverse=True).  `out` may be x."""
    if plan is None:
        raise ValueError("plan must be a RopePlan")
    hx, (B, L, H, D) = _heads(x, "x")
    out, hy = _output(out, x, "out", x.dtype)
    pos, pos_batch = _positions(plan, positions, B, L, x.device)
    _call("axial_rope", x.device, plan._h, hx, hy, B, L, D, pos, pos_batch, 1 if inverse else 0)
    return out


def _weights(q_weight, k_weight, D, dev):
    """The weights' common type."""
    dtype = None
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is None:
            continue
        if not isinstance(w, torch.Tensor) or w.dtype not in _TYPES or dtype not in (None, w.dtype):
            raise ValueError("the weights must be bf16 or fp32 tensors of one type")
        dtype = w.dtype
        _expect(w, name, dtype, (D,), dev)
    return _TYPES[dtype] if dtype is not None else ORBIT_OUT_F32


def _key(q, k, B, L, D):
    """k's rows, which share q's batches, tokens and head size but not its number of heads."""
    hk, (Bk, Lk, _, Dk) = _heads(k, "k", dtype=q.dtype)
    if (Bk, Lk, Dk) != (B, L, D) or k.dim() != q.dim() or k.device != q.device:
        raise ValueError(f"k must have q's batches, tokens, head size and device, got {tuple(k.shape)} beside {tuple(q.shape)}")
    return hk


def qk_norm_rope(plan: RopePlan, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, q_weight: torch.Tensor = None,
                 k_weight: torch.Tensor = None, eps: float = 1e-6, out_dtype: torch.dtype = None, q_out: torch.Tensor = None,
                 k_out: torch.Tensor = None):
    """(q, k), each head divided by sqrt(mean(x^2) + eps), multiplied by the weight [D] and turned as by axial_rope.
    plan = None (with positions = None): the norms alone; k = None: q alone.  q_out and k_out may be q and k."""
    hq, (B, L, H, D) = _heads(q, "q")
    if out_dtype is None:
        out_dtype = q.dtype if q_out is None else q_out.dtype
    if out_dtype not in _TYPES:
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    q_out, hqo = _output(q_out, q, "q_out", out_dtype)
    hk = hko = None
    if k is not None:
        hk = _key(q, k, B, L, D)
        k_out, hko = _output(k_out, k, "k_out", out_dtype)
    elif k_weight is not None or k_out is not None:
        raise ValueError("k_weight or k_out is given without k")
    pos, pos_batch = _positions(plan, positions, B, L, q.device)
    w_dtype = _weights(q_weight, k_weight, D, q.device)
    _call("qk_norm_rope", q.device, plan and plan._h, hq, hk, hqo, hko, B, L, D, pos, pos_batch, _ptr(q_weight), _ptr(k_weight),
          w_dtype, eps)
    return q_out, k_out


_workspace_bytes = {}


def _backward_workspace(D, dev):
    """Bytes that the weight gradients' partial sums take: fixed for a head size and device."""
    if (D, dev) not in _workspace_bytes:
        n = ctypes.c_size_t(0)
        with torch.cuda.device(dev):
            _check("qk_norm_rope_backward_workspace_size", lib().qk_norm_rope_backward_workspace_size(D, ctypes.byref(n)))
        _workspace_bytes[D, dev] = n.value
    return _workspace_bytes[D, dev]


def qk_norm_rope_backward(plan: RopePlan, dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          positions: torch.Tensor, q_weight: torch.Tensor = None, k_weight: torch.Tensor = None, eps: float = 1e-6,
                          q_grad: torch.Tensor = None, k_grad: torch.Tensor = None):
    """(q_grad, k_grad, q_weight_grad, k_weight_grad) from the gradients dq, dk of qk_norm_rope's outputs and from its
    inputs q and k: the first two in q's type, the weights' in fp32 (None for a weight that is None)."""
    hq, (B, L, H, D) = _heads(q, "q")
    hdq, _ = _heads(dq, "dq", q)
    q_grad, hqg = _output(q_grad, q, "q_grad", q.dtype)
    hk = hdk = hkg = None
    if k is not None:
        hk = _key(q, k, B, L, D)
        hdk, _ = _heads(dk, "dk", k, dq.dtype)
        k_grad, hkg = _output(k_grad, k, "k_grad", q.dtype)
    elif k_weight is not None or dk is not None or k_grad is not None:
        raise ValueError("dk, k_weight or k_grad is given without k")
    pos, pos_batch = _positions(plan, positions, B, L, q.device)
    w_dtype = _weights(q_weight, k_weight, D, q.device)
    dwq = None if q_weight is None else torch.empty((D,), dtype=torch.float32, device=q.device)
    dwk = None if k_weight is None else torch.empty((D,), dtype=torch.float32, device=q.device)
    ws, ws_bytes = None, 0
    if dwq is not None or dwk is not None:
        ws_bytes = _backward_workspace(D, q.device)
        ws = torch.empty((ws_bytes,), dtype=torch.uint8, device=q.device)
    _call("qk_norm_rope_backward", q.device, plan and plan._h, hdq, hdk, hq, hk, hqg, hkg, B, L, D, pos, pos_batch, _ptr(q_weight),
          _ptr(k_weight), w_dtype, eps, _ptr(dwq), _ptr(dwk), _ptr(ws), ws_bytes)
    return q_grad, k_grad, dwq, dwk
