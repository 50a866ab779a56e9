"""Low-rank adapters of many requests beside a projection that they share, with their gradients, in fp64 (test
infrastructure only).

Rows first .. end of a segment use adapter a: y = base + s_a (x A_a^T) B_a^T, with the first ranks[a] rows of A_a and
columns of B_a.  Rows without an adapter (-1) keep base.
"""

import numpy as np


def _segments(M, starts, adapters, ranks):
    for first, end, a in zip(starts, list(starts[1:]) + [M], adapters):
        if a >= 0 and ranks[a] > 0 and end > first:
            yield slice(first, end), a, ranks[a]


def lora_add(x, A, B, base, starts, adapters, ranks, scales):
    y = np.array(base, dtype=np.float64)
    for rows, a, r in _segments(len(y), starts, adapters, ranks):
        y[rows] += scales[a] * (x[rows] @ A[a, :r].T) @ B[a, :, :r].T
    return y


def lora_add_backward(dy, x, A, B, starts, adapters, ranks, scales):
    """(dx, dA, dB)."""
    dx, dA, dB = np.zeros(x.shape), np.zeros(A.shape), np.zeros(B.shape)
    for rows, a, r in _segments(len(x), starts, adapters, ranks):
        delta = scales[a] * dy[rows].T @ x[rows]           # gradient of the product B_a A_a
        dx[rows] = scales[a] * dy[rows] @ (B[a, :, :r] @ A[a, :r])
        dA[a, :r] += B[a, :, :r].T @ delta
        dB[a, :, :r] += delta @ A[a, :r].T
    return dx, dA, dB
