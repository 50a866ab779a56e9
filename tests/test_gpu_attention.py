"""GPU parity of attention and its gradients against the fp64 oracle, at the lengths, masks, layouts and values where they can
go wrong.

Bars, per value, with u = 2^-24 and h = 2^-8 (half a step of bf16).  A score is a sum of D exact products, off by
e = 10 sqrt(D) u scale sum|q k| (Higham and Mary, SIAM J. Sci. Comput. 2019, lambda = 10), and its exponential by E = 2 e + 32 u
(1 + |score| + |lse|) relative, the row's sum by the largest E of its keys.  So with E the row's largest:
    lse   E + 4 u |lse|
    o     half an ulp of its type + (h + 2 E + 10 sqrt(n) u) sum p |v|                (h: p enters the product in bf16)
    dv    half an ulp + (h + 2 E + 10 sqrt(rows) u) sum p |do|
    ds    p (2 E + h) |dp - delta| + p (10 sqrt(D) u (sum|do v| + sum|do o|) + sum|do| (error of o))
    dq, dk   half an ulp + scale sum (error of ds + 10 sqrt(n) u |ds|) |k|, |q|.
Probabilities, ds and products of them below the smallest normal number, t = 2^-126, may count as zeros (the exponential and the
matrix cores flush them): each term of a sum adds t (1 + its other factor) to o's and dv's bars, and to ds's error t (1 + |dp - delta|).
For example p = 1.7e-41 beside do = 0.8 is the whole of a dv at 150 x 400 pairs with scores of deviation 30.
"""

import math
import threading

import numpy as np
import pytest
import torch

import oracle
import paper_2607_02461_amd as oq
from paper_2607_02461_amd.launches import launches

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
H = 2.0 ** -8
T = 2.0 ** -126
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: H, F32: U}


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _within(name, got, ref, bar):
    got = _f64(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    over = np.abs(got - ref) / np.maximum(bar, 1e-300)
    assert got.size == 0 or over.max() <= 1.0, f"{name}: {over.max():.3f} of the bar at {np.unravel_index(over.argmax(), over.shape)}"


def _check_sequence(name, q, k, v, scale, causal, o, lse=None, do=None, grads=None):
    """One sequence's results against the oracle; q .. grads its rows of the tensors."""
    out_type, grad_type = o.dtype, BF16
    q, k, v = _f64(q), _f64(k), _f64(v)
    nq, heads, D = q.shape
    nk, G = k.shape[0], heads // k.shape[1]
    ref, ref_lse = oracle.attention(q, k, v, scale, causal)
    p, _ = oracle.attention_probabilities(q, k, scale, causal)
    grown = lambda n: 10 * math.sqrt(max(1, n)) * U  # noqa: E731
    bar_o, E = np.zeros(ref.shape), np.zeros((nq, heads))
    for h in range(heads):
        kh, vh = k[:, h // G], v[:, h // G]
        size = scale * np.abs(q[:, h]) @ np.abs(kh).T
        finite = np.where(np.isfinite(ref_lse[:, h]), np.abs(ref_lse[:, h]), 0.0)
        if nk:
            E[:, h] = (2 * grown(D) * size + 32 * U * (1 + np.abs(scale * q[:, h] @ kh.T))).max(axis=1) + 32 * U * finite
        bar_o[:, h] = (H + 2 * E[:, h:h + 1] + grown(nk)) * (p[h] @ np.abs(vh)) + T * (1 + np.abs(vh)).sum(0)
    _within(name + " o", o, ref, HALF[out_type] * np.abs(ref) + bar_o)
    if lse is not None:
        got = lse.double().cpu().numpy()
        live = np.isfinite(ref_lse)
        assert np.array_equal(np.isneginf(got), ~live), name
        assert (np.abs(got[live] - ref_lse[live]) <= E[live] + 4 * U * np.abs(ref_lse[live])).all(), name
    if grads is None:
        return
    do = _f64(do)
    dq, dk, dv = oracle.attention_backward(do, q, k, v, scale, causal)
    bars = [HALF[grad_type] * np.abs(t) for t in (dq, dk, dv)]
    for h in range(heads):
        qh, kh, vh, gh, at = q[:, h], k[:, h // G], v[:, h // G], do[:, h], h // G
        dp, delta = gh @ vh.T, (gh * ref[:, h]).sum(1, keepdims=True)
        e = E[:, h:h + 1]
        err = p[h] * ((2 * e + H) * np.abs(dp - delta) + grown(D) * (np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(ref[:, h])).sum(1, keepdims=True))
                      + (np.abs(gh) * (HALF[out_type] * np.abs(ref[:, h]) + bar_o[:, h])).sum(1, keepdims=True))
        err += T * (1 + np.abs(dp - delta))
        ds = p[h] * np.abs(dp - delta)
        bars[0][:, h] += scale * ((err + grown(nk) * ds) @ np.abs(kh) + nk * T)
        bars[1][:, at] += scale * ((err + grown(nq * G) * ds).T @ np.abs(qh) + nq * T)
        bars[2][:, at] += (p[h] * (H + 2 * e + grown(nq * G))).T @ np.abs(gh) + T * (1 + np.abs(gh)).sum(0)
    for n, got, want, bar in zip(("dq", "dk", "dv"), grads, (dq, dk, dv), bars):
        _within(f"{name} {n}", got, want, bar)


class Batch:
    """Sequences with random heads, in one of the layouts they have in use."""

    def __init__(self, q_lengths, k_lengths, heads, kv_heads, D, causal, seed=0, layout="dense", sharp=1.0, **starts):
        self.ql, self.kl = list(q_lengths), list(q_lengths if k_lengths is None else k_lengths)
        self.plan = oq.attention_plan(q_lengths, k_lengths, heads=heads, kv_heads=kv_heads, causal=causal, **starts)
        self.qs = starts.get("q_starts") or list(np.cumsum(self.ql) - self.ql)
        self.ks = starts.get("k_starts") or (self.qs if k_lengths is None else list(np.cumsum(self.kl) - self.kl))
        self.causal, self.scale = causal, sharp * D ** -0.5
        Mq, Mk = (max([s + n for s, n in zip(ss, nn)] + [0]) for ss, nn in ((self.qs, self.ql), (self.ks, self.kl)))
        g = torch.Generator().manual_seed(seed)
        make = lambda m, n: torch.randn((m, n, D), generator=g).to(BF16).to(DEV)  # noqa: E731
        q, k, v, do = make(Mq, heads), make(Mk, kv_heads), make(Mk, kv_heads), make(Mq, heads)
        if layout == "fused":        # queries, keys and values of one projection side by side
            m = max(Mq, Mk)
            whole = torch.full((m, heads + 2 * kv_heads, D), float("nan"), dtype=BF16, device=DEV)
            views = whole[:Mq, :heads], whole[:Mk, heads:heads + kv_heads], whole[:Mk, heads + kv_heads:]
            for to, t in zip(views, (q, k, v)):
                to.copy_(t)
            q, k, v = views
        elif layout == "heads":      # [heads, tokens, D] in memory
            q, k, v, do = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v, do))
        elif layout == "padded":     # heads of D + 8 values, tokens apart
            def pad(t):
                whole = torch.full((t.shape[0], t.shape[1] + 1, D + 8), float("nan"), dtype=BF16, device=DEV)
                whole[:, :-1, 8:] = t
                return whole[:, :-1, 8:]
            q, k, v, do = (pad(t) for t in (q, k, v, do))
        self.q, self.k, self.v, self.do = q, k, v, do
        self.lse = torch.full((Mq, heads), float("nan"), device=DEV)

    def forward(self, **kw):
        return oq.attention(self.plan, self.q, self.k, self.v, scale=self.scale, lse=self.lse, **kw)

    def backward(self, o, **kw):
        return oq.attention_backward(self.plan, self.do, self.q, self.k, self.v, o, self.lse, scale=self.scale, **kw)

    def check(self, o, grads=None):
        for i, (qs, nq, ks, nk) in enumerate(zip(self.qs, self.ql, self.ks, self.kl)):
            a, b = slice(qs, qs + nq), slice(ks, ks + nk)
            _check_sequence(f"sequence {i}", self.q[a], self.k[b], self.v[b], self.scale, self.causal, o[a], self.lse[a], self.do[a],
                            None if grads is None else (grads[0][a], grads[1][b], grads[2][b]))


# lengths of one and of tiles' edges, queries without keys and keys without queries, groups that do and do not divide a tile
CASES = [
    ([1], [1], 1, 1, 128), ([1], [64], 3, 3, 64), ([7], [65], 2, 1, 8), ([63, 64, 65], [64, 63, 65], 2, 2, 128), ([127, 128, 129], None, 4, 2, 64),
    ([0, 5, 0, 40], [9, 0, 0, 41], 4, 4, 96), ([300], [20], 2, 2, 80), ([20], [300], 6, 2, 128), ([33, 1, 257], [500, 130, 256], 10, 2, 40),
    ([5, 90], [333, 2], 7, 1, 128), ([2], [700], 96, 1, 24), ([130], [129], 70, 1, 16), ([1] * 5, [1, 31, 32, 33, 1000], 16, 2, 128), ([520], None, 3, 3, 112),
]


@pytest.mark.parametrize("ql,kl,heads,kv_heads,D", CASES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("layout", ["dense", "fused"])
def test_attention_and_gradients(ql, kl, heads, kv_heads, D, causal, layout):
    b = Batch(ql, kl, heads, kv_heads, D, causal, 1, layout)
    o = b.forward()
    assert o.dtype == BF16 and o.shape == b.q.shape
    b.check(o, b.backward(o))


@pytest.mark.parametrize("D,n", [(40, 60), (64, 700), (128, 60), (96, 512)])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_of_values_alike(D, n, causal):
    """Values alike, and keys: what the output's rounding takes from delta, e0 <= sum|do| (error of o), is many times what sets ds
    apart, and e0 sum p k many times dq.  The kernel finds delta again from p and dp, off by (2 E + 10 sqrt(n) u) sum p |dp| and the
    products' error; a bf16 rounding of what e0 leaves in ds and in the products that take it off is 2 h p e0."""
    heads = 2
    b = Batch([n], None, heads, heads, D, causal, 31)
    b.v.mul_(0.05).add_(1.0)
    b.k.add_(1.0)
    o = b.forward()
    dq, dk, _ = b.backward(o)
    q, k, v, do = (_f64(t) for t in (b.q, b.k, b.v, b.do))
    ref, _ = oracle.attention(q, k, v, b.scale, causal)
    p, _ = oracle.attention_probabilities(q, k, b.scale, causal)
    want = oracle.attention_backward(do, q, k, v, b.scale, causal)
    bars = [H * np.abs(t) for t in want[:2]]
    grown = lambda m: 10 * math.sqrt(m) * U  # noqa: E731
    for h in range(heads):
        qh, kh, vh, gh = q[:, h], k[:, h], v[:, h], do[:, h]
        scores, dp, delta = b.scale * qh @ kh.T, gh @ vh.T, (gh * ref[:, h]).sum(1, keepdims=True)
        lse = np.log(np.where(p[h] > 0, np.exp(scores), 0).sum(1))
        E = (2 * grown(D) * (b.scale * np.abs(qh) @ np.abs(kh).T) + 32 * U * (1 + np.abs(scores))).max(1, keepdims=True) + 32 * U * np.abs(lse)[:, None]
        products = grown(D) * (np.abs(gh) @ np.abs(vh).T).max(1, keepdims=True)
        e0 = (np.abs(gh) * (2 * H + 2 * E + grown(n)) * (p[h] @ np.abs(vh))).sum(1, keepdims=True)
        again = (2 * E + grown(n)) * (p[h] * np.abs(dp)).sum(1, keepdims=True)
        err = p[h] * ((2 * E + H) * np.abs(dp - delta) + 2 * products + again + 2 * H * e0) + T * (1 + np.abs(dp - delta))
        ds = p[h] * (np.abs(dp - delta) + e0)
        bars[0][:, h] += b.scale * ((err + grown(n) * ds) @ np.abs(kh) + n * T)
        bars[1][:, h] += b.scale * ((err + grown(n) * ds).T @ np.abs(qh) + n * T)
    _within("dq", dq, want[0], bars[0])
    _within("dk", dk, want[1], bars[1])


@pytest.mark.parametrize("layout", ["heads", "padded"])
@pytest.mark.parametrize("D", [64, 128])
def test_layouts_and_fp32_results(layout, D):
    b = Batch([70, 150], [200, 90], 6, 2, D, True, 2, layout)
    o = b.forward(out_dtype=F32)
    assert o.dtype == F32
    b.check(o, b.backward(o))
    whole = torch.zeros((220, 7, D + 8), dtype=BF16, device=DEV)
    out = whole[:, 1:, 8:]
    assert b.forward(out=out) is out and torch.equal(out, o.to(BF16)) and not whole[:, 0].any() and not whole[..., :8].any()


@pytest.mark.parametrize("rows,keys,heads,kv_heads,causal,ways", [
    (1, 5000, 8, 2, True, ["attention_few_kernel<128>", "attention_join_kernel<128>"]),       # single token, its keys divided
    (1, 100, 8, 2, True, ["attention_few_kernel<128>"]),
    (40, 3000, 4, 2, True, ["attention_kernel<128,4>", "attention_join_kernel<128>"]),           # a chunk of new tokens
    (1100, 1100, 4, 4, True, ["attention_kernel<128,4>", "attention_join_kernel<128>"]),         # a prompt that leaves compute units idle
    (1300, 1300, 4, 4, False, ["attention_kernel<128,4>", "attention_join_kernel<128>"]),
    (500, 500, 4, 4, False, ["attention_kernel<128,4>"]),                                        # short ones: a join would take longer
    (300, 70, 120, 120, False, ["attention_kernel<128,4>"]),
    (600, 8200, 180, 180, False, ["attention_kernel<128,8>"]),                                   # long, and enough of them: wide tiles
    (700, 16500, 172, 172, True, ["attention_kernel<128,8>"]),
])
def test_ways_of_the_forward_pass(rows, keys, heads, kv_heads, causal, ways):
    b = Batch([rows], [keys], heads, kv_heads, 128, causal, 3)
    o = b.forward()
    if heads * rows * keys < 1 << 28:
        b.check(o)
    else:                              # some heads of them, for the oracle's time
        for h in (0, 7, heads - 1):
            one = slice(h, h + 1)
            _check_sequence(f"head {h}", b.q[:, one], b.k[:, one], b.v[:, one], b.scale, causal, o[:, one], b.lse[:, one])
    assert [r.kernel for r in launches(lambda: b.forward(out=o))] == ways


@pytest.mark.parametrize("D,instance", [(24, 32), (64, 64), (96, 96), (128, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_wide_tiles_of_every_head_size_and_in_parts(D, instance, causal):
    # 64 sequences of up to 256 rows over one cache, one of them over many times the others' keys: its tile is divided, and parts
    # of 256 rows are joined
    heads, ql, most = 8, [256, 250, 130] + [256] * 61, (16500, 120000) if causal else (8200, 60000)
    kl = [most[0] + i for i in range(63)] + [most[1]]
    b = Batch(ql, kl, heads, heads, D, causal, 33, k_starts=[0] * 64)
    o = b.forward()
    for i in (0, 2, 63):
        nq, nk = ql[i], kl[i]
        for first, end in ((0, 20), (nq - 20, nq)):
            rows, keys = slice(b.qs[i] + first, b.qs[i] + end), slice(0, nk - (nq - end) if causal else nk)
            for h in (0, 7):
                one = slice(h, h + 1)
                _check_sequence(f"sequence {i} from {first}, head {h}", b.q[rows, one], b.k[keys, one], b.v[keys, one], b.scale, causal, o[rows, one],
                                b.lse[rows, one])
    assert [r.kernel for r in launches(lambda: b.forward(out=o))] == [f"attention_kernel<{instance},8>", f"attention_join_kernel<{instance}>"]
    assert torch.equal(b.forward(), o)


def test_a_long_clip_against_sampled_rows():
    # 32760 tokens: rows from the beginning, a tile's edges and the end, forward and backward
    n, heads, D = 32760, 2, 128
    b = Batch([n], None, heads, heads, D, False, 34)
    o = b.forward()
    dq, dk, dv = b.backward(o)
    rows = [0, 1, 127, 128, 20000, n - 1]
    _check_sequence("rows", b.q[rows], b.k, b.v, b.scale, False, o[rows], b.lse[rows])
    # dq of those rows alone: as if they were all the queries that there are (their bars do not depend on other rows)
    q, k, v, do = (_f64(t) for t in (b.q[rows], b.k, b.v, b.do[rows]))
    ref, lse = oracle.attention(q, k, v, b.scale)
    p, _ = oracle.attention_probabilities(q, k, b.scale, False)
    want = oracle.attention_backward(do, q, k, v, b.scale)[0]
    grown = lambda m: 10 * math.sqrt(m) * U  # noqa: E731
    for h in range(heads):
        qh, kh, vh, gh = q[:, h], k[:, h], v[:, h], do[:, h]
        dp, delta = gh @ vh.T, (gh * ref[:, h]).sum(1, keepdims=True)
        E = (2 * grown(D) * (b.scale * np.abs(qh) @ np.abs(kh).T) + 32 * U * (1 + np.abs(b.scale * qh @ kh.T))).max(1, keepdims=True) + 32 * U * np.abs(lse[:, h:h + 1])
        off_o = HALF[BF16] * np.abs(ref[:, h]) + (H + 2 * E + grown(n)) * (p[h] @ np.abs(vh)) + T * (1 + np.abs(vh)).sum(0)
        err = p[h] * ((2 * E + H) * np.abs(dp - delta) + grown(D) * (np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(ref[:, h])).sum(1, keepdims=True))
                      + (np.abs(gh) * off_o).sum(1, keepdims=True)) + T * (1 + np.abs(dp - delta))
        bar = HALF[BF16] * np.abs(want[:, h]) + b.scale * ((err + grown(n) * p[h] * np.abs(dp - delta)) @ np.abs(kh) + n * T)
        _within(f"dq, head {h}", dq[rows, h], want[:, h], bar)
    # every row of p sums to 1, so the sum of dv over keys is that of do; each dv is off by half an ulp and 2 h of its terms
    off = HALF[BF16] * dv.double().abs().sum(0) + 2.1 * H * b.do.double().abs().sum(0)
    assert ((dv.double().sum(0) - b.do.double().sum(0)).abs() <= off).all()


@pytest.mark.parametrize("rows,keys,heads,kv_heads,causal,joins", [
    (900, 60, 2, 2, False, 1), (60, 900, 4, 2, True, 1), (600, 600, 4, 1, True, 2), (200, 200, 64, 64, True, 0)])
def test_ways_of_the_backward_pass(rows, keys, heads, kv_heads, causal, joins):
    b = Batch([rows], [keys], heads, kv_heads, 64, causal, 4)
    o = b.forward()
    grads = b.backward(o)
    b.check(o, grads)
    ran = [r.kernel for r in launches(lambda: b.backward(o, q_grad=grads[0], k_grad=grads[1], v_grad=grads[2]))]
    assert sum("join" in r for r in ran) == joins, ran


def test_gradients_against_differences():
    b = Batch([9], [12], 2, 1, 16, True, 5)
    o = b.forward(out_dtype=F32)
    grads = b.backward(o)
    r = np.random.default_rng(1)
    values = [_f64(t) for t in (b.q, b.k, b.v)]
    along = [r.standard_normal(t.shape) for t in values]

    def loss(step):
        q, k, v = (t + step * d for t, d in zip(values, along))
        return float((oracle.attention(q, k, v, b.scale, True)[0] * _f64(b.do)).sum())

    want = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = sum(float((_f64(g) * d).sum()) for g, d in zip(grads, along))
    # each gradient's value is within 4 H of its terms; the terms of this sum are of the size of their root sum of squares
    size = math.sqrt(sum(float(((_f64(g) * d) ** 2).sum()) for g, d in zip(grads, along)))
    assert abs(got - want) <= 10 * 4 * H * size


@pytest.mark.parametrize("sharp", [0.01, 30.0])
def test_flat_and_sharp_rows(sharp):
    # 30: maxima that rise by many times the slack from tile to tile, rows of almost one key
    b = Batch([150], [400], 4, 2, 128, True, 6, sharp=sharp)
    o = b.forward()
    b.check(o, b.backward(o))


@pytest.mark.parametrize("scale,size", [(2.0 ** -100, 1.0), (2.0 ** 100, 2.0 ** -101)])
def test_smallest_and_large_scales(scale, size):
    b = Batch([90], [130], 4, 2, 64, True, 32, sharp=scale * 8.0)
    assert b.scale == scale
    b.q.mul_(size)
    o = b.forward()
    b.check(o, b.backward(o))


def test_scores_that_rise_and_fall_along_the_keys():
    # the running maximum rises at every tile, or is the first key's; both after and before keys with no weight
    b = Batch([40], [640], 1, 1, 64, False, 7)
    for first, last in ((-40, 40), (40, -40)):
        b.k[:, :, 0] = torch.linspace(first, last, 640, device=DEV).to(BF16)[:, None]
        b.q[:, :, 0] = 8.0
        o = b.forward()
        b.check(o, b.backward(o))


def test_padded_batches_and_tokens_of_no_sequence():
    # three samples padded to 200 tokens; the padding holds values that are not finite, in inputs and in outputs' places
    ql, kl = [130, 1, 200], [77, 200, 3]
    b = Batch(ql, kl, 4, 2, 128, False, 8, q_starts=[0, 200, 400], k_starts=[0, 200, 400])
    want, plain = b.forward(), b.backward(b.forward())
    b.check(want, plain)
    dead_q = torch.ones(b.q.shape[0], dtype=torch.bool, device=DEV)
    dead_k = torch.ones(b.k.shape[0], dtype=torch.bool, device=DEV)
    for s, n in zip(b.qs, ql):
        dead_q[s:s + n] = False
    for s, n in zip(b.ks, kl):
        dead_k[s:s + n] = False
    assert not want[dead_q].any() and not any(g[d].any() for g, d in zip(plain, (dead_q, dead_k, dead_k)))   # new tensors: zeros
    b.q[dead_q], b.do[dead_q], b.k[dead_k], b.v[dead_k] = float("nan"), float("inf"), float("nan"), float("-inf")
    out = torch.full_like(want, 5.0)
    b.lse.fill_(9.0)
    b.forward(out=out)
    assert torch.equal(out[~dead_q], want[~dead_q]) and (out[dead_q] == 5.0).all() and (b.lse[dead_q] == 9.0).all()
    grads = [torch.full_like(t, 6.0) for t in (b.q, b.k, b.v)]
    b.backward(out, q_grad=grads[0], k_grad=grads[1], v_grad=grads[2])
    for g, p, d in zip(grads, plain, (dead_q, dead_k, dead_k)):
        assert torch.equal(g[~d], p[~d]) and (g[d] == 6.0).all()


def test_rows_that_see_nothing_and_keys_that_nothing_sees():
    b = Batch([200], [70], 4, 2, 128, True, 9)
    o = b.forward()
    dq, dk, dv = b.backward(o)
    assert not o[:130].any() and torch.isneginf(b.lse[:130]).all() and not dq[:130].any()
    b.check(o, (dq, dk, dv))
    none = oq.attention_plan([50, 0], [0, 90], heads=2, causal=False)
    q, k = torch.randn((50, 2, 64), device=DEV).to(BF16), torch.randn((90, 2, 64), device=DEV).to(BF16)
    lse = torch.zeros((50, 2), device=DEV)
    o = oq.attention(none, q, k, k, lse=lse)
    assert not o.any() and torch.isneginf(lse).all()
    assert not any(g.any() for g in oq.attention_backward(none, q, q, k, k, o, lse))


def test_sequences_that_share_keys():
    # several requests over one prefix, one of them in the middle of it
    kl, ks = [400, 400, 100], [0, 0, 150]
    b = Batch([1, 60, 3], kl, 4, 2, 128, False, 10, k_starts=ks)
    b.check(b.forward())
    with pytest.raises(oq.OrbitError, match="key in common"):
        b.backward(b.forward())


def test_values_that_are_not_finite_stay_in_their_sequence():
    b = Batch([100, 130, 1], [100, 130, 90], 4, 2, 128, True, 11)
    o = b.forward()
    want, grads = o.clone(), b.backward(o)
    b.k[150, 0], b.v[160, 1], b.q[105, 3] = float("nan"), float("inf"), float("nan")
    got = b.forward()
    clean = torch.ones(231, dtype=torch.bool, device=DEV)
    clean[100:230] = False
    assert torch.equal(got[clean], want[clean])
    assert not torch.isfinite(got[150:230, :2]).any() and not torch.isfinite(got[105, 3]).any() and not torch.isfinite(got[160:230, 2:]).any()
    again = b.backward(got)
    for a, c, n in zip(again, grads, (231, 320, 320)):
        rows = torch.ones(n, dtype=torch.bool, device=DEV)
        rows[100:230] = False
        assert torch.equal(a[rows], c[rows])


def test_the_same_bits_each_time_and_beside_other_sequences():
    b = Batch([300, 1, 64], [300, 900, 64], 8, 2, 128, True, 12)
    o = b.forward()
    grads = b.backward(o)
    for _ in range(3):
        assert torch.equal(b.forward(), o) and all(torch.equal(x, y) for x, y in zip(b.backward(o), grads))


def test_streams_devices_and_graphs():
    b = Batch([300, 1, 77], [300, 2000, 64], 8, 2, 128, True, 13)

    def both():
        o = b.forward()
        return (o,) + tuple(b.backward(o))

    want = both()
    torch.cuda.synchronize()
    got = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                lse = torch.empty_like(b.lse)
                o = oq.attention(b.plan, b.q, b.k, b.v, scale=b.scale, lse=lse)
                got.append((o,) + tuple(oq.attention_backward(b.plan, b.do, b.q, b.k, b.v, o, lse, scale=b.scale)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for g in got for a, c in zip(g, want))
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append(both())
    g = torch.Generator().manual_seed(14)
    for _ in range(3):
        for t in (b.q, b.k, b.v, b.do):
            t.copy_(torch.randn(t.shape, generator=g).to(BF16))
        for i in (0, 1):
            graphs[i].replay()
            torch.cuda.synchronize()
        fresh = both()
        assert all(torch.equal(a, c) for h in held for a, c in zip(h, fresh))


@pytest.mark.parametrize("D", [64, 128])
def test_inputs_that_are_broadcast(D):
    # heads, and tokens, that share their memory, given and in place of the other operands one after the other
    b = Batch([70, 130], [90, 200], 8, 2, D, True, 35)
    for name in ("q", "k", "v", "do"):
        for at in ((slice(None), slice(0, 1)), (slice(0, 1),)):
            whole = getattr(b, name)
            view = whole[at].expand(whole.shape)
            assert 0 in view.stride()
            results = []
            for t in (view, view.contiguous()):
                setattr(b, name, t)
                o = b.forward()
                results.append((o, b.lse.clone()) + tuple(b.backward(o)))
            setattr(b, name, whole)
            assert all(torch.equal(x, y) for x, y in zip(*results)), name


def test_calls_of_two_threads():
    b = Batch([200, 1, 33], [300, 2000, 64], 8, 2, 64, True, 36)
    o = b.forward()
    want = (o,) + tuple(b.backward(o))
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    lse = torch.empty_like(b.lse)
                    out = oq.attention(b.plan, b.q, b.k, b.v, scale=b.scale, lse=lse)
                    got = (out,) + tuple(oq.attention_backward(b.plan, b.do, b.q, b.k, b.v, out, lse, scale=b.scale))
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(x, y) for x, y in zip(got, want))
        except BaseException as e:  # noqa: BLE001 (of a thread: raised below)
            errors.append(e)

    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_many_short_sequences_and_many_heads():
    r = np.random.default_rng(2)
    ql, kl = [int(n) for n in r.integers(0, 5, 300)], [int(n) for n in r.integers(0, 40, 300)]
    b = Batch(ql, kl, 5, 5, 64, True, 15)
    o = b.forward()
    b.check(o, b.backward(o))


def test_long_rows_against_sampled_rows():
    # keys and rows whose offsets pass 2^32 bytes: tokens that lie far apart
    n, D, apart = 3000, 64, 1 << 20
    whole = torch.empty((n, apart), dtype=BF16, device=DEV)           # 6.3 GB
    g = torch.Generator().manual_seed(16)
    views = [whole[:, 64 * i:64 * (i + 2)].unflatten(1, (2, 64)) for i in (0, 2, 4, 6, 8, 10, 12, 14)]
    for t in views[:4]:
        t.copy_(torch.randn((n, 2, D), generator=g).to(BF16))
    q, k, v, do = views[:4]
    plan = oq.attention_plan([n], heads=2, causal=True)
    lse = torch.empty((n, 2), device=DEV)
    o = oq.attention(plan, q, k, v, out=views[4], lse=lse)
    grads = oq.attention_backward(plan, do, q, k, v, o, lse, q_grad=views[5], k_grad=views[6], v_grad=views[7])
    dense = [t.contiguous() for t in (q, k, v, do)]
    lse2 = torch.empty_like(lse)
    o2 = oq.attention(plan, *dense[:3], lse=lse2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    for a, c in zip(grads, oq.attention_backward(plan, dense[3], *dense[:3], o2, lse2)):
        assert torch.equal(a, c)
    rows = slice(n - 3, n)
    _check_sequence("the last rows", q[rows], k, v, D ** -0.5, True, o[rows], lse[rows])


def test_refusals():
    plan = oq.attention_plan([10], [20], heads=4, kv_heads=2)
    q, k = torch.zeros((10, 4, 64), dtype=BF16, device=DEV), torch.zeros((20, 2, 64), dtype=BF16, device=DEV)
    lse = torch.zeros((10, 4), device=DEV)
    for call, word in ((lambda: oq.attention(None, q, k, k), "plan"), (lambda: oq.attention(plan, q.cpu(), k, k), "GPU"), (lambda: oq.attention(plan, q.float(), k, k), "bfloat16"),
                       (lambda: oq.attention(plan, q[:9], k, k), "at least 10"), (lambda: oq.attention(plan, q, k[:19], k), "at least 20"),
                       (lambda: oq.attention(plan, q[:, :2], k, k), "heads"), (lambda: oq.attention(plan, q, k, k[..., :32]), "v must be"),
                       (lambda: oq.attention(plan, q, k, k, out=q[:, :1].expand(10, 4, 64)), "overlap"), (lambda: oq.attention(plan, q, k, k, out_dtype=torch.float16), "out_dtype"),
                       (lambda: oq.attention(plan, q, k, k, lse=lse[:, :2]), "lse"), (lambda: oq.attention(plan, q[0], k, k), "q must be"),
                       (lambda: oq.attention(plan, q.transpose(1, 2), k, k), "q must be"),
                       (lambda: oq.attention_backward(plan, q[..., :32], q, k, k, q, lse), "dout"), (lambda: oq.attention_backward(plan, q, q, k, k, q, lse.double()), "lse"),
                       (lambda: oq.attention_backward(plan, q, q, k, k, q, lse, k_grad=k.float()), "k_grad")):
        with pytest.raises(ValueError, match=word):
            call()
    for call, word in ((lambda: oq.attention(plan, q, k, k, scale=0.0), "scale"), (lambda: oq.attention(plan, q, k, k, out=q), "lies on"),
                       (lambda: oq.attention(plan, torch.zeros((10, 4, 136), dtype=BF16, device=DEV), *2 * [torch.zeros((20, 2, 136), dtype=BF16, device=DEV)]), "head size"),
                       (lambda: oq.attention(plan, torch.zeros((10, 4, 68), dtype=BF16, device=DEV)[..., 4:], k, k), "16 bytes")):
        with pytest.raises(oq.OrbitError, match=word):
            call()
