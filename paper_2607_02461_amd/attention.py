"""Attention over packed sequences of any lengths, grouped heads, causal or not, forward and backward.

    plan = attention_plan(q_lengths, k_lengths, heads=32, kv_heads=8, causal=True)   # once for a batch
    out = attention(plan, q, k, v)                     # q [tokens, 32, D], k and v [tokens, 8, D], sequences behind each other

Heads are bf16 tensors [token, head, D] whose last dimension is contiguous: views of the fused projection's output and of
qk_norm_rope's (batches flattened into tokens) are taken as they lie.  A padded batch gives its sequences' starts.
"""

import ctypes
import math

import numpy as np
import torch

from . import _c_void_p, _call, _check, _expect, _ptr, lib
from .attention_input import _TYPES, _pack_heads, _rows_apart


class AttentionPlan:
    """Handle of a batch's sequences of queries and keys."""

    def __init__(self, handle, heads, kv_heads, queries, keys):
        self._h, self._destroy = handle, lib().attention_plan_destroy
        self.heads, self.kv_heads = heads, kv_heads
        # (tokens behind the last one, tokens of all sequences): they are equal where the sequences leave none out
        self._queries, self._keys = queries, keys
        self._bytes = {}

    @property
    def handle(self):
        return self._h

    def upload(self, device=None):
        """Copies the lists to `device` (default: the current one), as Plan.upload."""
        with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
            _check("attention_plan_upload", lib().attention_plan_upload(self._h))
        return self

    def _workspace(self, D, backward, dev):
        """(a new workspace or None, its bytes); the plan and the head size alone decide them."""
        if (D, backward) not in self._bytes:
            n = ctypes.c_size_t(0)
            _check("attention_workspace_size", lib().attention_workspace_size(self._h, D, backward, ctypes.byref(n)))
            self._bytes[D, backward] = n.value
        n = self._bytes[D, backward]
        return torch.empty((n,), dtype=torch.uint8, device=dev) if n else None, n

    def __del__(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None


def _numbers(v, name):
    v = np.asarray(v)
    if v.ndim != 1 or (v.size and v.dtype.kind not in "iu") or (v.size and v.dtype.kind == "u" and int(v.max()) >= 1 << 63):
        raise ValueError(f"{name} must be a list of whole numbers")
    return np.ascontiguousarray(v, dtype=np.int64)


def _sequences(lengths, starts, name):
    """(starts, lengths) of sequences behind each other where no starts are given."""
    lengths = _numbers(lengths, f"{name}_lengths")
    if starts is None:
        return np.cumsum(lengths) - lengths, lengths
    starts = _numbers(starts, f"{name}_starts")
    if starts.shape != lengths.shape:
        raise ValueError(f"{name}_starts and {name}_lengths must be of one length")
    return starts, lengths


def _extent(starts, lengths):
    live = lengths > 0
    return int((starts + lengths)[live].max(initial=0)), int(lengths.sum())


def attention_plan(q_lengths, k_lengths=None, *, heads: int, kv_heads: int = None, causal: bool = False, q_starts=None,
                   k_starts=None) -> AttentionPlan:
    """The plan of a batch of sequences: queries and keys of each (k_lengths = None: as many keys as queries, in the same
    places), `heads` query heads over kv_heads key heads (default: as many).  With `causal`, query i of n_q sees the first
    i + 1 + n_k - n_q keys of its sequence.  Sequences lie behind each other, or at q_starts and k_starts."""
    qs, ql = _sequences(q_lengths, q_starts, "q")
    if k_lengths is None:
        if k_starts is not None:
            raise ValueError("k_starts are given without k_lengths")
        ks, kl = qs, ql
    else:
        ks, kl = _sequences(k_lengths, k_starts, "k")
    if ql.shape != kl.shape:
        raise ValueError("q_lengths and k_lengths must be of one length")
    heads, kv_heads = int(heads), int(heads if kv_heads is None else kv_heads)
    if not all(-(1 << 31) <= n < 1 << 31 for n in (heads, kv_heads)):
        raise ValueError("heads and kv_heads must be 32-bit numbers")
    out = _c_void_p()
    _check("attention_plan", lib().attention_plan(ql.size, qs.ctypes.data, ql.ctypes.data, ks.ctypes.data, kl.ctypes.data, heads, kv_heads,
                                                  int(bool(causal)), ctypes.byref(out)))
    return AttentionPlan(out, heads, kv_heads, _extent(qs, ql), _extent(ks, kl))


def _heads(t, name, heads, tokens, D=None, dev=None, dtypes=(torch.bfloat16,)):
    """t's rows for the library: [at least `tokens`, heads, D]."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[0] < tokens or (D and shape[2] != D):
        raise ValueError(f"{name} must be [at least {tokens} tokens, {heads} heads, {'D' if D is None else D}], got {tuple(shape)}")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on {dev}")
    sl, sh, sd = t.stride()
    if sd != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    return _pack_heads(t.data_ptr(), 0, sl, sh, heads, _TYPES[t.dtype])


def _output(out, like, name, extent, dtype):
    """(out, its rows): the caller's output, checked, or a new one of `like`'s shape, zeros where no sequence has a token."""
    if out is None:
        whole = extent[0] == extent[1] == like.shape[0]
        out = (torch.empty_like if whole else torch.zeros_like)(like, dtype=dtype, memory_format=torch.contiguous_format)
        _, H, D = like.shape
        return out, _pack_heads(out.data_ptr(), 0, H * D, D, H, _TYPES[dtype])
    rows = _heads(out, name, like.shape[1], extent[0], like.shape[2], like.device, (dtype,))
    if out.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}, got {tuple(out.shape)}")
    _rows_apart(out, name)
    return out, rows


def _inputs(plan, q, k, v):
    """(D, rows of q, k and v)."""
    if not isinstance(plan, AttentionPlan):
        raise ValueError("plan must be an AttentionPlan")
    hq = _heads(q, "q", plan.heads, plan._queries[0])
    D, dev = q.shape[2], q.device
    return D, hq, _heads(k, "k", plan.kv_heads, plan._keys[0], D, dev), _heads(v, "v", plan.kv_heads, plan._keys[0], D, dev)


def attention(plan: AttentionPlan, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float = None,
              out: torch.Tensor = None, out_dtype: torch.dtype = None, lse: torch.Tensor = None) -> torch.Tensor:
    """softmax(scale q k^T) v for each query over the keys that the plan lets it see: q [tokens, heads, D], k and v [tokens,
    kv_heads, D], scale 1 / sqrt(D) if none is given.  The output is bf16 (or fp32 with out_dtype: not rounded at the end, but
    of probabilities that enter the product with v in bf16, 2^-8 relative, all the same) in q's shape: zeros where a query sees no key; tokens of no sequence are left as they were in `out`, zeros in a new tensor.  `lse`: an fp32 tensor
    [tokens, heads] that receives the logarithms of the rows' sums for the backward pass."""
    D, hq, hk, hv = _inputs(plan, q, k, v)
    if out_dtype is None:
        out_dtype = torch.bfloat16 if out is None else out.dtype
    if out_dtype not in _TYPES:
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    out, ho = _output(out, q, "out", plan._queries, out_dtype)
    if lse is not None:
        _expect(lse, "lse", torch.float32, (q.shape[0], plan.heads), q.device)
    ws, ws_bytes = plan._workspace(D, 0, q.device)
    _call("attention", q.device, plan._h, hq, hk, hv, ho, D, 1 / math.sqrt(D) if scale is None else scale, _ptr(lse), _ptr(ws), ws_bytes)
    return out


def attention_backward(plan: AttentionPlan, dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, scale: float = None, q_grad: torch.Tensor = None, k_grad: torch.Tensor = None,
                       v_grad: torch.Tensor = None):
    """(q_grad, k_grad, v_grad), bf16 in the shapes of q, k and v, from dout, the gradient of attention's output in bf16, its
    inputs, its output and its lse.  Probabilities and their gradients enter the products in bf16.  Tokens of no sequence are left as they were in gradients that are given (views of a
    fused projection's gradient, for example), zeros in new ones.  The plan's sequences share no keys."""
    D, hq, hk, hv = _inputs(plan, q, k, v)
    dev = q.device
    hg = _heads(dout, "dout", plan.heads, plan._queries[0], D, dev)
    ho = _heads(out, "out", plan.heads, plan._queries[0], D, dev, (torch.bfloat16, torch.float32))
    _expect(lse, "lse", torch.float32, (q.shape[0], plan.heads), dev)
    q_grad, hdq = _output(q_grad, q, "q_grad", plan._queries, torch.bfloat16)
    k_grad, hdk = _output(k_grad, k, "k_grad", plan._keys, torch.bfloat16)
    v_grad, hdv = _output(v_grad, v, "v_grad", plan._keys, torch.bfloat16)
    ws, ws_bytes = plan._workspace(D, 1, dev)
    _call("attention_backward", dev, plan._h, hg, hq, hk, hv, ho, lse.data_ptr(), hdq, hdk, hdv, D,
          1 / math.sqrt(D) if scale is None else scale, _ptr(ws), ws_bytes)
    return q_grad, k_grad, v_grad
