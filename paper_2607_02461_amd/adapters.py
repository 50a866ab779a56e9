"""Low-rank adapters of many requests beside a projection that they share, forward and backward.

    plan = lora_plan(M, starts, adapters, ranks, scales)      # once for a batch of requests
    Y = orbit_qlinear_ws(...)                                 # the shared projection
    lora_add(plan, X, A, B, Y, out=Y)                         # + scale_a (X A_a^T) B_a^T for each request's rows
"""

import ctypes

import numpy as np
import torch

from . import ORBIT_OUT_BF16, ORBIT_OUT_F32, _c_void_p, _call, _check, _expect, _output, _ptr, _rows, lib


class LoraPlan:
    """Handle of a batch's segments of rows and of their adapters' ranks and scales."""

    def __init__(self, handle, rows, adapters):
        self._h, self._destroy = handle, lib().lora_plan_destroy
        self.rows, self.adapters = rows, adapters
        self._bytes = {}

    @property
    def handle(self):
        return self._h

    def upload(self, device=None):
        """Copies the lists to `device` (default: the current one), as Plan.upload."""
        with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
            _check("lora_plan_upload", lib().lora_plan_upload(self._h))
        return self

    def _workspace(self, K, N, R, backward, dev):
        """(a new workspace or None, its bytes); the plan and the sizes alone decide them."""
        key = (K, N, R, backward, dev)
        if key not in self._bytes:
            n = ctypes.c_size_t(0)
            with torch.cuda.device(dev):
                _check("lora_add_workspace_size", lib().lora_add_workspace_size(self._h, K, N, R, backward, ctypes.byref(n)))
            self._bytes[key] = n.value
        n = self._bytes[key]
        return torch.empty((n,), dtype=torch.uint8, device=dev) if n else None, n

    def __del__(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None


def lora_plan(M: int, starts, adapters, ranks, scales) -> LoraPlan:
    """The plan of M rows: segment s is rows starts[s] .. starts[s + 1] - 1 (the last one ends at M) and uses adapter
    adapters[s], -1 for none; adapter a has rank ranks[a] and scale scales[a]."""
    starts, adapters, ranks, scales = (np.asarray(v) for v in (starts, adapters, ranks, scales))
    for name, v, kinds in (("starts", starts, "iu"), ("adapters", adapters, "iu"), ("ranks", ranks, "iu"), ("scales", scales, "iuf")):
        if v.ndim != 1 or (v.size and v.dtype.kind not in kinds):
            raise ValueError(f"{name} must be a list of numbers")
        if v.size and v.dtype.kind in "iu" and not (-(1 << 31) <= int(v.min()) and int(v.max()) < 1 << 31):
            raise ValueError(f"{name} must be 32-bit numbers")
    if starts.shape != adapters.shape or ranks.shape != scales.shape:
        raise ValueError("starts and adapters must be of one length, ranks and scales too")
    starts, adapters = np.ascontiguousarray(starts, dtype=np.int64), np.ascontiguousarray(adapters, dtype=np.int32)
    ranks, scales = np.ascontiguousarray(ranks, dtype=np.int32), np.ascontiguousarray(scales, dtype=np.float32)
    out = _c_void_p()
    _check("lora_plan", lib().lora_plan(M, starts.size, starts.ctypes.data, adapters.ctypes.data, ranks.size, ranks.ctypes.data,
                                        scales.ctypes.data, ctypes.byref(out)))
    return LoraPlan(out, int(M), int(ranks.size))


def _operands(plan, X, A, B):
    """(K, N, R, X's row stride, device)."""
    if not isinstance(plan, LoraPlan):
        raise ValueError("plan must be a LoraPlan")
    M, K, ldx, dev = _rows(X, "X")
    if M != plan.rows:
        raise ValueError(f"X has {M} rows, the plan {plan.rows}")
    if not isinstance(A, torch.Tensor) or A.dim() != 3 or not isinstance(B, torch.Tensor) or B.dim() != 3:
        raise ValueError("A and B must be 3-D tensors")
    R, N = A.shape[1], B.shape[1]
    _expect(A, "A", torch.bfloat16, (plan.adapters, R, K), dev)
    _expect(B, "B", torch.bfloat16, (plan.adapters, N, R), dev)
    return K, N, R, max(ldx, K) if M <= 1 else ldx, dev


def _addend(base, name, M, N, dtype, dev):
    """(pointer, row stride) of a wide input."""
    if not isinstance(base, torch.Tensor) or base.device != dev or base.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} tensor on {dev}")
    if tuple(base.shape) != (M, N) or base.stride(1) != 1 or (M > 1 and base.stride(0) < N):
        raise ValueError(f"{name} must have the shape ({M}, {N}) and contiguous rows")
    return base.data_ptr(), max(base.stride(0), N)


def lora_add(plan: LoraPlan, X: torch.Tensor, A: torch.Tensor, B: torch.Tensor, base: torch.Tensor, out: torch.Tensor = None,
             h: torch.Tensor = None) -> torch.Tensor:
    """base + scale_a (X A_a^T) B_a^T, a the adapter of each row's segment: X bf16 [M, K], A bf16 [adapters, R, K],
    B bf16 [adapters, N, R], base fp32 or bf16 [M, N], the shared projection's output.  `out` may be base.  `h`: an fp32
    tensor [M, R] that receives X A^T for the backward pass."""
    K, N, R, ldx, dev = _operands(plan, X, A, B)
    M = plan.rows
    if not isinstance(base, torch.Tensor) or base.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("base must be a bf16 or fp32 tensor")
    pb, ldb = _addend(base, "base", M, N, base.dtype, dev)
    out, ldy = _output(out, M, N, base.dtype, dev)
    if h is not None:
        _expect(h, "h", torch.float32, (M, R), dev)
    ws, ws_bytes = plan._workspace(K, N, R, 0, dev)
    _call("lora_add", dev, plan._h, X.data_ptr(), ldx, A.data_ptr(), B.data_ptr(), K, N, R, pb, ldb,
          ORBIT_OUT_BF16 if base.dtype == torch.bfloat16 else ORBIT_OUT_F32, out.data_ptr(), ldy, _ptr(h),
          _ptr(ws), ws_bytes)
    return out


def lora_add_backward(plan: LoraPlan, dY: torch.Tensor, X: torch.Tensor, A: torch.Tensor, B: torch.Tensor, h: torch.Tensor,
                      base: torch.Tensor = None, out: torch.Tensor = None):
    """(dX bf16 [M, K], dA fp32 [adapters, R, K], dB fp32 [adapters, N, R]) from dY, the gradient of lora_add's output in
    bf16, its inputs and its h.  dX is added to `base`, bf16 [M, K], where that is given (the gradient that X has from
    the projection); `out` receives dX and may be base.  The gradient of lora_add's base is dY."""
    K, N, R, ldx, dev = _operands(plan, X, A, B)
    M = plan.rows
    pd, ldd = _addend(dY, "dY", M, N, torch.bfloat16, dev)
    _expect(h, "h", torch.float32, (M, R), dev)
    pb, ldb = (None, 0) if base is None else _addend(base, "base", M, K, torch.bfloat16, dev)
    out, lddx = _output(out, M, K, torch.bfloat16, dev)
    dA = torch.empty(A.shape, dtype=torch.float32, device=dev)
    dB = torch.empty(B.shape, dtype=torch.float32, device=dev)
    ws, ws_bytes = plan._workspace(K, N, R, 1, dev)
    _call("lora_add_backward", dev, plan._h, pd, ldd, X.data_ptr(), ldx, A.data_ptr(), B.data_ptr(), h.data_ptr(), K, N, R, pb, ldb,
          out.data_ptr(), lddx, dA.data_ptr(), dB.data_ptr(), _ptr(ws), ws_bytes)
    return out, dA, dB
