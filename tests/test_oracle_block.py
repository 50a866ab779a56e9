"""The oracle of layer norms and attention: gradients against differences, closed forms, rows that see nothing."""

import numpy as np
import pytest

import oracle


def _differences(loss, values, grads, step=1e-5):
    for i, (value, grad) in enumerate(zip(values, grads)):
        for at in range(value.size):
            d = np.zeros(value.size)
            d[at] = step
            d = d.reshape(value.shape)
            up, down = ([v + s * d if j == i else v for j, v in enumerate(values)] for s in (1, -1))
            assert (loss(*up) - loss(*down)) / (2 * step) == pytest.approx(grad.flat[at], rel=1e-6, abs=1e-8)


def test_layer_norm_gradients_against_differences():
    r = np.random.default_rng(1)
    x, dy, g, b = r.standard_normal((2, 3, 7)) + 2.0, r.standard_normal((2, 3, 7)), r.standard_normal(7), r.standard_normal(7)
    dx, dg, db = oracle.layer_norm_backward(dy, x, g, eps=0.1)
    _differences(lambda x, g, b: float(np.sum(dy * oracle.layer_norm(x, g, b, eps=0.1))), (x, g, b), (dx, dg.sum((0, 1)), db.sum((0, 1))))


def test_layer_norm_closed_forms():
    assert np.allclose(oracle.layer_norm(np.array([[1.0, 3.0]]), eps=0.0), [[-1.0, 1.0]])
    assert np.array_equal(oracle.layer_norm(np.full((1, 4), 5.0), 3.0, 2.0), np.full((1, 4), 2.0))   # no variance: the offset
    x = np.random.default_rng(2).standard_normal((5, 64))
    y = oracle.layer_norm(x, eps=0.0)
    assert np.allclose(y.mean(-1), 0.0) and np.allclose((y * y).mean(-1), 1.0)
    assert np.allclose(oracle.layer_norm(3.0 * x + 100.0, eps=0.0), y)


@pytest.mark.parametrize("nq,nk,H,Hk,causal", [(3, 4, 2, 1, False), (4, 3, 2, 2, True), (2, 5, 4, 2, True)])
def test_attention_gradients_against_differences(nq, nk, H, Hk, causal):
    r = np.random.default_rng(3)
    q, k, v, do = (r.standard_normal(s) for s in ((nq, H, 3), (nk, Hk, 3), (nk, Hk, 3), (nq, H, 3)))
    grads = oracle.attention_backward(do, q, k, v, 0.7, causal)
    _differences(lambda q, k, v: float(np.sum(do * oracle.attention(q, k, v, 0.7, causal)[0])), (q, k, v), grads)


def test_attention_closed_forms():
    r = np.random.default_rng(4)
    k, v = r.standard_normal((6, 1, 4)), r.standard_normal((6, 1, 4))
    o, lse = oracle.attention(np.zeros((2, 2, 4)), k, v, 1.0)              # equal scores: the mean
    assert np.allclose(o, v.mean(0)[None]) and np.allclose(lse, np.log(6.0))
    o, lse = oracle.attention(1e4 * k[3:4], k, v, 1.0)                     # one score above all: its value
    best = int(np.argmax(k[:, 0] @ k[3, 0]))
    assert np.allclose(o[0, 0], v[best, 0])
    q = r.standard_normal((6, 1, 4))
    whole, _ = oracle.attention(q, k, v, 0.5, causal=True)
    for i in range(6):                                                     # token by token over what there is so far
        assert np.allclose(whole[i:i + 1], oracle.attention(q[i:i + 1], k[:i + 1], v[:i + 1], 0.5, causal=True)[0])


def test_queries_that_see_no_key():
    r = np.random.default_rng(5)
    q, k, v, do = (r.standard_normal(s) for s in ((5, 1, 4), (2, 1, 4), (2, 1, 4), (5, 1, 4)))
    o, lse = oracle.attention(q, k, v, 1.0, causal=True)
    assert not o[:3].any() and np.isneginf(lse[:3]).all() and np.allclose(o[3, 0], v[0, 0]) and np.isfinite(lse[3:]).all()
    dq, dk, dv = oracle.attention_backward(do, q, k, v, 1.0, causal=True)
    assert not dq[:4].any() and np.allclose(dv[0] + dv[1], do[3] + do[4]) and np.isfinite(dk).all()
    assert not oracle.attention(q, k[:0], v[:0], 1.0)[0].any()
