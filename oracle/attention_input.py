"""Rotary positions with several axes and the RMS norms of query and key heads, with their gradients, in fp64
(test infrastructure only).

A head's first 2 P values are P pairs: (2p, 2p + 1), or (p, P + p) with `halves`.  Axis by axis, the pairs turn by
position * theta^(-2 j / dim), j counting the axis's own dim / 2 pairs.  As complex numbers, z' = z exp(i angle).
The norm divides a head by sqrt(mean(x^2) + eps) and multiplies by a weight; it comes before the turn.
"""

import numpy as np


def rope_angles(dims, positions, theta=10000.0):
    """Angles [..., P] of positions [..., axes]."""
    positions = np.asarray(positions, dtype=np.float64)
    parts = [positions[..., a:a + 1] * theta ** (-2.0 * np.arange(d // 2) / d) for a, d in enumerate(dims)]
    return np.concatenate(parts, axis=-1)


def rope_turn(x, angles, halves=False, sign=1.0):
    """x [B, L, H, D] turned by sign * angles [B or 1, L, P]."""
    x = np.asarray(x, dtype=np.float64)
    P = angles.shape[-1]
    first, second = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    z = (x[..., first] + 1j * x[..., second]) * np.exp(1j * sign * angles)[..., None, :]
    out = x.copy()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def qk_norm_rope(x, angles, weight=None, eps=1e-6, halves=False):
    """One tensor of heads; angles = None: the norm alone."""
    x = np.asarray(x, dtype=np.float64)
    n = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, dtype=np.float64))
    return n if angles is None else rope_turn(n, angles, halves)


def qk_norm_rope_backward(dy, x, angles, weight=None, eps=1e-6, halves=False):
    """(dx, dweight): with s = mean(x^2) + eps and n_i = x_i w_i / sqrt(s), the chain rule term by term."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    D = x.shape[-1]
    w = np.ones(D) if weight is None else np.asarray(weight, dtype=np.float64)
    g = dy if angles is None else rope_turn(dy, angles, halves, -1.0)
    s = np.mean(x * x, axis=-1, keepdims=True) + eps
    through_s = np.sum(g * w * x, axis=-1, keepdims=True) * (-0.5) * s ** -1.5   # d loss / d s
    dx = g * w * s ** -0.5 + through_s * 2.0 * x / D
    return dx, np.sum(g * x * s ** -0.5, axis=(0, 1, 2))
