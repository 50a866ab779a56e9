"""Attention of one sequence's query heads over key heads that groups of them share, and its gradients, in fp64 (test
infrastructure only).

q [n_q, H, D], k and v [n_k, H_k, D]: head h reads key head h // (H / H_k).  causal: query i sees keys j <= i + n_k - n_q.  A
query that sees no key has zeros, and an lse of -inf.
"""

import numpy as np


def _visible(nq, nk, causal):
    return np.arange(nk)[None, :] <= np.arange(nq)[:, None] + (nk - nq) if causal else np.ones((nq, nk), dtype=bool)


def probabilities(q, k, scale, causal):
    """(p [H, n_q, n_k], lse [n_q, H])."""
    nq, H, _ = q.shape
    nk, Hk, _ = k.shape
    p, lse = np.zeros((H, nq, nk)), np.full((nq, H), -np.inf)
    see = _visible(nq, nk, causal)
    some = see.any(axis=1)
    for h in range(H):
        s = np.where(see, scale * (q[:, h] @ k[:, h // (H // Hk)].T), -np.inf)[some]
        if s.size:
            m = s.max(axis=1, keepdims=True)
            e = np.exp(s - m)
            p[h][some] = e / e.sum(axis=1, keepdims=True)
            lse[some, h] = m[:, 0] + np.log(e.sum(axis=1))
    return p, lse


def attention(q, k, v, scale, causal=False):
    """(o [n_q, H, D], lse [n_q, H])."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    G = q.shape[1] // k.shape[1]
    p, lse = probabilities(q, k, scale, causal)
    return np.stack([p[h] @ v[:, h // G] for h in range(q.shape[1])], axis=1), lse


def attention_backward(do, q, k, v, scale, causal=False):
    """(dq, dk, dv): through the softmax's Jacobian, diag(p) - p p^T."""
    do, q, k, v = (np.asarray(t, dtype=np.float64) for t in (do, q, k, v))
    G = q.shape[1] // k.shape[1]
    p, _ = probabilities(q, k, scale, causal)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(q.shape[1]):
        dp = do[:, h] @ v[:, h // G].T
        ds = p[h] * dp - p[h] * (p[h] * dp).sum(axis=1, keepdims=True)
        dq[:, h] = scale * ds @ k[:, h // G]
        dk[:, h // G] += scale * ds.T @ q[:, h]
        dv[:, h // G] += p[h].T @ do[:, h]
    return dq, dk, dv
