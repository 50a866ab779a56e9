"""The oracle of the rotary positions and of the query and key norms: properties of the rotation, and the gradients
against differences."""

import numpy as np
import pytest

import oracle


def _case(seed, B=2, L=3, H=2, D=16, dims=(4, 6, 2)):
    r = np.random.default_rng(seed)
    x, dy = r.standard_normal((2, B, L, H, D))
    return x, dy, r.uniform(0.5, 1.5, D), oracle.rope_angles(dims, r.integers(0, 50, (B, L, len(dims))))


@pytest.mark.parametrize("halves", [False, True])
def test_turn_keeps_lengths_and_turns_back(halves):
    x, _, _, angles = _case(1)
    y = oracle.rope_turn(x, angles, halves)
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-14)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    assert np.allclose(oracle.rope_turn(y, angles, halves, -1.0), x, rtol=0, atol=1e-14)


@pytest.mark.parametrize("halves", [False, True])
def test_products_depend_on_differences_of_positions(halves):
    r = np.random.default_rng(2)
    dims = (4, 8)
    q, k = r.standard_normal((2, 1, 1, 1, 12))

    def product(a, b):
        turned = [oracle.rope_turn(v, oracle.rope_angles(dims, np.array([[p]])), halves) for v, p in ((q, a), (k, b))]
        return float(np.sum(turned[0] * turned[1]))

    assert product((5, 9), (2, 30)) == pytest.approx(product((13, 11), (10, 32)), rel=1e-12)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("turned", [False, True])
def test_gradients_against_differences(halves, turned):
    x, dy, w, angles = _case(3)
    angles = angles if turned else None
    eps = 1e-3

    def loss(x, w):
        return float(np.sum(dy * oracle.qk_norm_rope(x, angles, w, eps, halves)))

    dx, dw = oracle.qk_norm_rope_backward(dy, x, angles, w, eps, halves)
    step = 1e-5
    for at in np.random.default_rng(4).permutation(x.size)[:40]:
        d = np.zeros(x.size)
        d[at] = step
        d = d.reshape(x.shape)
        assert (loss(x + d, w) - loss(x - d, w)) / (2 * step) == pytest.approx(dx.flat[at], rel=1e-6, abs=1e-8)
    for at in range(w.size):
        d = np.zeros(w.size)
        d[at] = step
        assert (loss(x, w + d) - loss(x, w - d)) / (2 * step) == pytest.approx(dw[at], rel=1e-6, abs=1e-8)
