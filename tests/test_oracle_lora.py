"""The oracle of the low-rank adapters: its gradients against differences, rows without an adapter, rows beyond ranks."""

import numpy as np
import pytest

import oracle


def test_gradients_against_differences():
    r = np.random.default_rng(1)
    M, K, N, R, n = 7, 6, 5, 4, 3
    x, dy = r.standard_normal((M, K)), r.standard_normal((M, N))
    A, B, base = r.standard_normal((n, R, K)), r.standard_normal((n, N, R)), r.standard_normal((M, N))
    batch = dict(starts=[1, 3, 3, 5], adapters=[2, 1, -1, 2], ranks=[4, 1, 3], scales=[1.0, 0.5, 2.0])
    grads = oracle.lora_add_backward(dy, x, A, B, **batch)

    def loss(x, A, B):
        return float(np.sum(dy * oracle.lora_add(x, A, B, base, **batch)))

    step = 1e-5
    for i, (value, grad) in enumerate(zip((x, A, B), grads)):
        for at in range(value.size):
            d = np.zeros(value.size)
            d[at] = step
            d = d.reshape(value.shape)
            up, down = ([v + s * d if j == i else v for j, v in enumerate((x, A, B))] for s in (1, -1))
            assert (loss(*up) - loss(*down)) / (2 * step) == pytest.approx(grad.flat[at], rel=1e-6, abs=1e-8)
    assert not grads[1][0].any() and not grads[2][0].any()          # an adapter without rows
    assert not grads[1][1, 1:].any() and not grads[2][1, :, 1:].any()   # beyond the rank
    assert not grads[0][0].any()                                    # a row before the first segment


def test_rows_without_an_adapter_keep_the_base():
    r = np.random.default_rng(2)
    x, A, B, base = (r.standard_normal(s) for s in ((6, 4), (1, 2, 4), (1, 3, 2), (6, 3)))
    y = oracle.lora_add(x, A, B, base, [2, 4], [0, -1], [2], [1.5])
    assert np.array_equal(y[:2], base[:2]) and np.array_equal(y[4:], base[4:])
    assert np.allclose(y[2:4], base[2:4] + 1.5 * x[2:4] @ (B[0] @ A[0]).T)
