"""Layer norm of rows with gain and offset, and its gradients, in fp64 (test infrastructure only).

y = (x - mean) / sqrt(var + eps) * g + b over the last axis; g and b broadcast against x.
"""

import numpy as np


def layer_norm(x, g=1.0, b=0.0, eps=1e-6):
    x = np.asarray(x, dtype=np.float64)
    d = x - x.mean(-1, keepdims=True)
    return d / np.sqrt((d * d).mean(-1, keepdims=True) + eps) * g + b


def layer_norm_backward(dy, x, g=1.0, eps=1e-6):
    """(dx, each row's terms of dg, each row's terms of db): the chain rule through the mean and the variance."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    N = x.shape[-1]
    d = x - x.mean(-1, keepdims=True)
    s = (d * d).mean(-1, keepdims=True) + eps
    h = dy * g
    through_s = (h * d).sum(-1, keepdims=True) * (-0.5) * s ** -1.5        # d loss / d s
    dd = h * s ** -0.5 + through_s * 2.0 * d / N                           # d loss / d (x - mean)
    return dd - dd.mean(-1, keepdims=True), dy * d * s ** -0.5, dy
