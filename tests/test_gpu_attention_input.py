"""GPU parity of the rotary positions and of the query and key norms against the fp64 oracle, at the layouts, sizes
and values where they can go wrong.

Bars, per value: a result is computed in fp32 and rounded once to its type, so |y - ref| <= half an ulp of the type
(2^-8 |ref| in bf16, 2^-24 |ref| in fp32) + 32 u S, with u = 2^-24 and S the size of what is added up: the pair's
length sqrt(a^2 + b^2) for a turn, and for dx, r (|g w| + |x| r^2 mean|g w x|), both of the pair's lengths.  32 u
covers the table's rounding, the norm's sum of at most 512 squares (pairwise over lanes, 8 in a row), the root and
five products.  Weight gradients are sums of n terms: 10 sqrt(n) u sum|terms| (Higham and Mary, SIAM J. Sci. Comput.
2019, lambda = 10) + 32 u sum|terms|.
"""

import re

import numpy as np
import pytest
import torch

import oracle
import paper_2607_02461_amd as oq
from paper_2607_02461_amd import launches as launches_module

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
EPS = 1e-6
BF16, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _pair_length(x, P, halves):
    """Per value, the length of the pair it belongs to (its own magnitude beyond the pairs)."""
    out = np.abs(x)
    first, second = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out[..., first] = out[..., second] = np.hypot(x[..., first], x[..., second])
    return out


def _check(name, got, ref, size, dtype):
    got, bar = _f64(got), HALF_ULP[dtype] * np.abs(ref) + 32 * U * size
    over = np.abs(got - ref) / np.maximum(bar, 1e-300)
    assert np.isfinite(got).all(), f"{name}: not finite"
    assert got.size == 0 or over.max() <= 1.0, f"{name}: {over.max():.3f} of the bar at {np.unravel_index(over.argmax(), over.shape)}"


def _rows(shape, dtype, seed, layout="dense"):
    """Heads [B, L, H, D] with channels of different size, in one of the layouts they have in use."""
    B, L, H, D = shape
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(shape, generator=g) * torch.exp(torch.randn((H, D), generator=g))).to(dtype).to(DEV)
    if layout == "fused":      # q or k of [B, L, 3, H, D]
        whole = torch.full((B, L, 3, H, D), float("nan"), dtype=dtype, device=DEV)
        whole[:, :, 1] = x
        return whole[:, :, 1]
    if layout == "heads":      # [B, H, L, D] in memory
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "padded":     # rows of D + 8 values
        whole = torch.full((B, L, H, D + 8), float("nan"), dtype=dtype, device=DEV)
        whole[..., 8:] = x
        return whole[..., 8:]
    return x


def _plan_and_positions(dims, B, L, seed, halves, shared=True, lengths=None):
    lengths = lengths or [40] * len(dims)
    g = torch.Generator().manual_seed(seed)
    pos = torch.stack([torch.randint(0, n, (L,) if shared else (B, L), generator=g) for n in lengths], dim=-1).to(torch.int32)
    angles = oracle.rope_angles(dims, pos.numpy() if not shared else pos.numpy()[None])
    return oq.rope_plan(dims, lengths, halves=halves), pos.to(DEV), angles


SHAPES = [
    ((1, 1, 1, 8), (8,)), ((1, 1, 24, 128), (16, 56, 56)), ((2, 5, 3, 128), (44, 42, 42)), ((1, 77, 40, 128), (64, 64)),
    ((3, 13, 7, 64), (16, 24, 24)), ((2, 9, 5, 96), (16, 24, 24)), ((2, 6, 4, 80), (40, 40)), ((1, 11, 2, 256), (64, 96, 96)),
    ((2, 3, 1, 512), (2, 4, 6, 8, 10, 12, 14, 456)), ((1, 301, 13, 16), (8,)), ((5, 2, 65, 32), (4, 12, 8)), ((1, 3, 2, 24), (10, 6)),
]


@pytest.mark.parametrize("shape,dims", SHAPES)
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("inverse", [False, True])
def test_axial_rope(shape, dims, halves, dtype, inverse):
    B, L, H, D = shape
    plan, pos, angles = _plan_and_positions(dims, B, L, 1, halves)
    x = _rows(shape, dtype, 2)
    ref = oracle.rope_turn(_f64(x), angles, halves, -1.0 if inverse else 1.0)
    y = oq.axial_rope(plan, x, pos, inverse=inverse)
    assert y.dtype == dtype and y.shape == x.shape
    _check("axial_rope", y, ref, _pair_length(_f64(x), sum(dims) // 2, halves), dtype)


@pytest.mark.parametrize("shape,dims", SHAPES)
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
def test_qk_norm_rope(shape, dims, halves, dtype, out):
    B, L, H, D = shape
    plan, pos, angles = _plan_and_positions(dims, B, L, 3, halves, shared=False)
    q, k = _rows(shape, dtype, 4), _rows((B, L, max(1, H // 3), D), dtype, 5)
    g = torch.Generator().manual_seed(6)
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(dtype).to(DEV) for _ in range(2))
    got = oq.qk_norm_rope(plan, q, k, pos, wq, wk, eps=EPS, out_dtype=out)
    for name, x, w, y in (("q", q, wq, got[0]), ("k", k, wk, got[1])):
        n = oracle.qk_norm_rope(_f64(x), None, _f64(w), EPS)
        assert y.dtype == out and y.shape == x.shape
        _check(name, y, oracle.rope_turn(n, angles, halves), _pair_length(n, sum(dims) // 2, halves), out)


def _check_backward(name, got, dw, dy, x, w, angles, P, halves, eps=EPS):
    B, L, H, D = x.shape
    dy, x64, w64 = _f64(dy), _f64(x), np.ones(D) if w is None else _f64(w)
    ref, dw_ref = oracle.qk_norm_rope_backward(dy, x64, angles, w64, eps, halves)
    g = dy if angles is None else oracle.rope_turn(dy, angles, halves, -1.0)
    size = _pair_length(g, P, halves) * np.abs(w64)
    r = 1 / np.sqrt(np.mean(x64 * x64, axis=-1, keepdims=True) + eps)
    size = r * (size + np.abs(x64) * r * r * np.mean(size * np.abs(x64), axis=-1, keepdims=True))
    _check(f"{name} grad", got, ref, size, x.dtype)
    if w is None:
        assert dw is None
        return
    terms = np.sum(_pair_length(g, P, halves) * np.abs(x64) * r, axis=(0, 1, 2))
    assert dw.dtype == F32
    bar = (10 * np.sqrt(B * L * H) + 32) * U * terms
    assert (np.abs(_f64(dw) - dw_ref) <= bar + 1e-300).all(), f"{name} weight grad"


@pytest.mark.parametrize("shape,dims", SHAPES)
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
def test_qk_norm_rope_backward(shape, dims, halves, dtype, grad):
    B, L, H, D = shape
    plan, pos, angles = _plan_and_positions(dims, B, L, 7, halves)
    Hk = max(1, H // 3)
    q, k, dq, dk = _rows(shape, dtype, 8), _rows((B, L, Hk, D), dtype, 9), _rows(shape, grad, 10), _rows((B, L, Hk, D), grad, 11)
    g = torch.Generator().manual_seed(12)
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(DEV) for _ in range(2))
    gq, gk, dwq, dwk = oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, wq, wk, eps=EPS)
    assert gq.dtype == dtype and gk.dtype == dtype
    _check_backward("q", gq, dwq, dq, q, wq, angles, sum(dims) // 2, halves)
    _check_backward("k", gk, dwk, dk, k, wk, angles, sum(dims) // 2, halves)


@pytest.mark.parametrize("layout", ["fused", "heads", "padded"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(layout, halves, dtype):
    # inputs as they lie in use, outputs too: what lies between an output's rows keeps its value
    shape, dims = (2, 19, 6, 64), (16, 24, 16)
    plan, pos, angles = _plan_and_positions(dims, 2, 19, 13, halves)
    q, k, dq, dk = (_rows(shape, dtype, s, layout) for s in (14, 15, 16, 17))
    w = torch.linspace(0.5, 2.0, 64, device=DEV)
    outs = []
    for _ in range(4):
        whole = torch.full((2, 19, 6, 80), 7.0, dtype=dtype, device=DEV)
        outs.append((whole, whole[..., 8:72]))
    oq.qk_norm_rope(plan, q, k, pos, w, None, eps=EPS, q_out=outs[0][1], k_out=outs[1][1])
    for x, weight, (_, y) in ((q, _f64(w), outs[0]), (k, None, outs[1])):
        n = oracle.qk_norm_rope(_f64(x), None, weight, EPS)
        _check(layout, y, oracle.rope_turn(n, angles, halves), _pair_length(n, 28, halves), dtype)
    _, _, dwq, dwk = oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, w, None, eps=EPS, q_grad=outs[2][1], k_grad=outs[3][1])
    _check_backward("q", outs[2][1], dwq, dq, q, w, angles, 28, halves)
    _check_backward("k", outs[3][1], dwk, dk, k, None, angles, 28, halves)
    for whole, _ in outs:
        assert (whole[..., :8] == 7.0).all() and (whole[..., 72:] == 7.0).all()


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place(halves, dtype):
    # H = 5 leaves lane groups of the last step without a head of their own
    shape, dims = (2, 33, 5, 96), (16, 24, 24)
    plan, pos, _ = _plan_and_positions(dims, 2, 33, 18, halves)
    q, k, dq, dk = (_rows(shape, dtype, s, "fused") for s in (19, 20, 21, 22))
    w = torch.linspace(0.5, 2.0, 96, device=DEV)
    want = oq.axial_rope(plan, q, pos)
    x = _rows(shape, dtype, 19, "fused")
    assert oq.axial_rope(plan, x, pos, out=x).data_ptr() == x.data_ptr() and torch.equal(x, want)
    want = oq.qk_norm_rope(plan, q, k, pos, w, w)
    back = oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, w, w)
    x, y = _rows(shape, dtype, 19, "fused"), _rows(shape, dtype, 20, "fused")
    oq.qk_norm_rope(plan, x, y, pos, w, w, q_out=x, k_out=y)
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])
    got = oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, w, w, q_grad=dq, k_grad=dk)
    assert all(torch.equal(a, b) for a, b in zip(got, back))


def test_norm_without_rotation_query_without_key_and_no_weights():
    q = _rows((2, 7, 3, 128), BF16, 23)
    y, none = oq.qk_norm_rope(None, q, None, None, eps=EPS)
    assert none is None
    n = oracle.qk_norm_rope(_f64(q), None, None, EPS)
    _check("norm", y, n, np.abs(n), BF16)
    dy = _rows((2, 7, 3, 128), BF16, 24)
    gq, gk, dwq, dwk = oq.qk_norm_rope_backward(None, dy, None, q, None, None, eps=EPS)
    assert gk is None and dwk is None
    _check_backward("q", gq, dwq, dy, q, None, None, 0, False)


def test_three_dimensions_are_one_batch():
    plan, pos, _ = _plan_and_positions((64, 64), 1, 9, 25, False)
    x = _rows((1, 9, 4, 128), BF16, 26)
    assert torch.equal(oq.axial_rope(plan, x[0], pos), oq.axial_rope(plan, x, pos)[0])


def test_broadcast_inputs():
    # one key for every batch and head, read in place; its gradient comes for each use
    plan, pos, angles = _plan_and_positions((16, 16), 3, 10, 27, False)
    k = _rows((1, 10, 1, 32), F32, 28).expand(3, 10, 4, 32)
    q, dq, dk = (_rows((3, 10, 4, 32), F32, s) for s in (29, 30, 31))
    w = torch.ones(32, device=DEV)
    _, y = oq.qk_norm_rope(plan, q, k, pos, w, w, eps=EPS)
    n = oracle.qk_norm_rope(_f64(k), None, None, EPS)
    _check("k", y, oracle.rope_turn(n, angles), _pair_length(n, 16, False), F32)
    _, gk, _, dwk = oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, w, w, eps=EPS)
    _check_backward("k", gk, dwk, dk, k, w, angles, 16, False)


def test_zero_rows_and_empty_tensors():
    plan, pos, _ = _plan_and_positions((64, 64), 1, 4, 32, False)
    w = torch.ones(128, device=DEV)
    z = torch.zeros((1, 4, 3, 128), dtype=BF16, device=DEV)
    dy = _rows((1, 4, 3, 128), BF16, 33)
    y, _ = oq.qk_norm_rope(plan, z, None, pos, w, eps=EPS)
    assert (y == 0).all()
    gq, _, dwq, _ = oq.qk_norm_rope_backward(plan, dy, None, z, None, pos, w, eps=EPS)
    assert torch.isfinite(gq).all() and (dwq == 0).all()
    e = z[:, :0]
    none = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    assert oq.axial_rope(plan, e, none).shape == e.shape
    y, k = oq.qk_norm_rope(plan, e, e, none, w, w)
    assert y.shape == e.shape and k.shape == e.shape
    _, _, dwq, dwk = oq.qk_norm_rope_backward(plan, e, e, e, e, none, w, w)
    assert (dwq == 0).all() and (dwk == 0).all()


@pytest.mark.parametrize("halves", [False, True])
def test_values_beyond_the_pairs_are_copied_whatever_they_are(halves):
    plan, pos, _ = _plan_and_positions((8, 8), 1, 3, 34, halves)
    x = _rows((1, 3, 2, 64), BF16, 35)
    x[0, 1, 1, 16:20] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.4e38], device=DEV)
    y = oq.axial_rope(plan, x, pos)
    assert torch.equal(y[..., 16:].view(torch.int16), x[..., 16:].view(torch.int16))
    assert torch.isfinite(y[..., :16]).all()


def test_a_row_that_is_not_finite_stays_alone():
    plan, pos, _ = _plan_and_positions((64, 64), 1, 6, 36, False)
    q = _rows((1, 6, 4, 128), BF16, 37)
    want, _ = oq.qk_norm_rope(plan, q, None, pos)
    q[0, 2, 1, 5] = float("nan")
    q[0, 4, 3, 100] = float("inf")
    got, _ = oq.qk_norm_rope(plan, q, None, pos)
    hit = torch.zeros((1, 6, 4), dtype=torch.bool, device=DEV)
    hit[0, 2, 1] = hit[0, 4, 3] = True
    assert torch.equal(got[~hit], want[~hit])
    assert torch.isnan(got[0, 2, 1]).all() and torch.isnan(got[0, 4, 3, 100])


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("where", [-1, 40, 2 ** 31 - 1, -2 ** 31])
def test_positions_without_angles_give_nan_on_their_axis_alone(halves, where):
    plan, pos, _ = _plan_and_positions((8, 16, 8), 1, 5, 38, halves)
    x = _rows((1, 5, 3, 40), F32, 39)
    want = oq.axial_rope(plan, x, pos)
    pos[3, 1] = where
    got = oq.axial_rope(plan, x, pos)
    hit = torch.zeros_like(x, dtype=torch.bool)
    pairs = torch.arange(4, 12, device=DEV)
    hit[:, 3, :, torch.cat([pairs, pairs + 16] if halves else [2 * pairs, 2 * pairs + 1])] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


def test_plan_from_angles():
    r = np.random.default_rng(40)
    angles = [r.uniform(-9, 9, (5, 6)), r.uniform(-9, 9, (3, 10))]
    plan = oq.rope_plan_from_angles(angles, halves=True)
    assert plan.dims == (12, 20) and plan.lengths == (5, 3)
    pos = np.array([[4, 0], [0, 2], [2, 1]], dtype=np.int32)
    x = _rows((1, 3, 2, 32), F32, 41)
    at = np.concatenate([angles[0][pos[:, 0]], angles[1][pos[:, 1]]], axis=1)[None]
    _check("angles", oq.axial_rope(plan, x, torch.from_numpy(pos).to(DEV)), oracle.rope_turn(_f64(x), at, True),
           _pair_length(_f64(x), 16, True), F32)


def test_far_positions():
    # an angle of 10^6 radians is exact to fp64's rounding in the table; formed in fp32 it would be off by 0.03
    plan = oq.rope_plan((8,), (1_000_001,))
    pos = torch.tensor([[1_000_000], [999_999]], dtype=torch.int32, device=DEV)
    x = _rows((1, 2, 2, 8), F32, 42)
    angles = oracle.rope_angles((8,), pos.cpu().numpy()[None])
    _check("far", oq.axial_rope(plan, x, pos), oracle.rope_turn(_f64(x), angles), _pair_length(_f64(x), 4, False), F32)


def test_weight_gradients_have_the_same_bits_every_time_and_at_many_rows():
    plan, pos, angles = _plan_and_positions((16, 24, 24), 2, 1500, 43, False)
    q, dq = _rows((2, 1500, 5, 64), BF16, 44), _rows((2, 1500, 5, 64), BF16, 45)
    w = torch.linspace(0.5, 2.0, 64, device=DEV)
    first = oq.qk_norm_rope_backward(plan, dq, dq, q, q, pos, w, w, eps=EPS)
    _check_backward("q", first[0], first[2], dq, q, w, angles, 32, False)
    assert torch.equal(first[2], first[3])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, oq.qk_norm_rope_backward(plan, dq, dq, q, q, pos, w, w, eps=EPS)))


@pytest.mark.parametrize("shape,stride", [((1, 70, 2, 64), (0, 2 ** 26 + 8, 64, 1)), ((2, 3, 2, 64), (64, 2 ** 31 + 8, 2 ** 30, 1))])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_beyond_32_bits(shape, stride, dtype):
    plan, pos, _ = _plan_and_positions((16, 24, 16), shape[0], shape[1], 13, False)
    q, dq = (_rows(shape, dtype, s) for s in (61, 62))
    w = torch.linspace(0.5, 2.0, 64, device=DEV)
    size = sum(n * (d - 1) for n, d in zip(stride, shape)) + 1

    def apart(t):
        return torch.empty(size, dtype=dtype, device=DEV).as_strided(shape, stride).copy_(t)

    far, out = apart(q), apart(torch.zeros_like(q))
    assert torch.equal(oq.axial_rope(plan, far, pos, out=out), oq.axial_rope(plan, q, pos))
    assert torch.equal(oq.qk_norm_rope(plan, far, far, pos, w, w, eps=EPS, q_out=out)[0], oq.qk_norm_rope(plan, q, q, pos, w, w, eps=EPS)[0])
    want = oq.qk_norm_rope_backward(plan, dq, dq, q, q, pos, w, w, eps=EPS)
    got = oq.qk_norm_rope_backward(plan, apart(dq), dq, far, q, pos, w, w, eps=EPS, q_grad=out)
    assert torch.equal(out, want[0]) and torch.equal(got[2], want[2])


def test_streams_and_graph_replays():
    plan, pos, _ = _plan_and_positions((64, 64), 2, 50, 46, False)
    w = torch.linspace(0.5, 2.0, 128, device=DEV)
    make = lambda s: [_rows((2, 50, 6, 128), BF16, s + i, "fused") for i in range(4)]  # noqa: E731

    def call(q, k, dq, dk):
        return oq.qk_norm_rope(plan, q, k, pos, w, w) + oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, w, w)

    stream = torch.cuda.Stream()
    inputs = make(50)
    want = call(*inputs)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = call(*inputs)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call(*inputs)
    for seed in (60, 70, 80):
        for to, new in zip(inputs, make(seed)):
            to.copy_(new)
        want = call(*inputs)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    plan, pos, _ = _plan_and_positions((64, 64), 2, 5, 47, False)
    x = _rows((2, 5, 3, 128), BF16, 48)
    w = torch.ones(128, device=DEV)

    def refused(call, *words):
        with pytest.raises((ValueError, oq.OrbitError)) as e:
            call()
        assert all(word in str(e.value) for word in words), str(e.value)

    refused(lambda: oq.axial_rope(None, x, pos), "plan")
    refused(lambda: oq.axial_rope(plan, x.cpu(), pos), "GPU")
    refused(lambda: oq.axial_rope(plan, x.half(), pos), "bf16 or fp32")
    refused(lambda: oq.axial_rope(plan, x[0, 0], pos), "[batch, token, head, D]")
    refused(lambda: oq.axial_rope(plan, x, pos.long()), "positions")
    refused(lambda: oq.axial_rope(plan, x, pos[:4]), "positions")
    refused(lambda: oq.axial_rope(plan, x, pos.t().contiguous().t()), "positions")
    refused(lambda: oq.axial_rope(plan, x, pos.cpu()), "positions")
    refused(lambda: oq.axial_rope(plan, x, None), "positions")
    refused(lambda: oq.axial_rope(plan, x[..., :64], pos), "rotates 128")
    refused(lambda: oq.axial_rope(plan, _rows((2, 5, 3, 132), BF16, 1)[..., :128], pos), "16 bytes")
    refused(lambda: oq.axial_rope(plan, _rows((2, 5, 3, 136), BF16, 1)[..., 4:132], pos), "16 bytes")
    refused(lambda: oq.axial_rope(plan, x.transpose(2, 3).contiguous().transpose(2, 3), pos), "contiguous")
    refused(lambda: oq.axial_rope(plan, x, pos, out=torch.empty_like(x, dtype=F32)), "out")
    refused(lambda: oq.axial_rope(plan, x, pos, out=torch.empty_like(x[:1]).expand(2, 5, 3, 128)), "overlap")
    refused(lambda: oq.axial_rope(plan, x, pos, out=x[:, :4]), "shape")
    refused(lambda: oq.qk_norm_rope(None, x, x, pos), "without a plan")
    refused(lambda: oq.qk_norm_rope(plan, x, x[:, :4], pos), "k must have")
    refused(lambda: oq.qk_norm_rope(plan, x, x.float(), pos), "k must be")
    refused(lambda: oq.qk_norm_rope(plan, x, None, pos, None, w), "without k")
    refused(lambda: oq.qk_norm_rope(plan, x, x, pos, w, w.to(BF16)), "one type")
    refused(lambda: oq.qk_norm_rope(plan, x, x, pos, w[:64], w), "q_weight")
    refused(lambda: oq.qk_norm_rope(plan, x, x, pos, w, w, eps=-1.0), "eps")
    refused(lambda: oq.qk_norm_rope(plan, x, x, pos, w, w, eps=float("nan")), "eps")
    refused(lambda: oq.qk_norm_rope(plan, x, x, pos, w, w, out_dtype=torch.float16), "out_dtype")
    refused(lambda: oq.qk_norm_rope_backward(plan, x, x.float(), x, x, pos, w, w), "dk")
    refused(lambda: oq.qk_norm_rope_backward(plan, x[:, :4], x, x, x, pos, w, w), "dq")
    refused(lambda: oq.qk_norm_rope_backward(plan, x, x, x, None, pos, w), "without k")
    refused(lambda: oq.qk_norm_rope(None, _rows((1, 1, 1, 20), BF16, 1)[..., :12], None, None), "head size 12")
    refused(lambda: oq.qk_norm_rope(None, _rows((1, 1, 1, 520), BF16, 1), None, None), "head size 520")


# --- large tensors: non-temporal loads and stores ---------------------------------------------------
def _turned(x, angles, halves, sign=1.0):
    """rope_turn in fp64 on the device."""
    P = angles.shape[-1]
    c, s = torch.cos(angles)[None, :, None], sign * torch.sin(angles)[None, :, None]
    first, second = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    y = x.clone()
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., first] * s + x[..., second] * c
    return y


def _device_pair_length(x, P, halves):
    out = x.abs()
    first, second = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out[..., first] = out[..., second] = torch.hypot(x[..., first], x[..., second])
    return out


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("D,dims", [(128, (16, 56, 56)), (160, (64, 64))])
def test_large_tensors(dtype, out, halves, D, dims):
    # above 160 MiB in and out
    size = {BF16: 2, F32: 4}
    H = 9
    L = (170 << 20) // (H * D * (size[dtype] + size[out])) + 3
    lengths = [L] * len(dims)
    plan = oq.rope_plan(dims, lengths, halves=halves)
    g = torch.Generator(device=DEV).manual_seed(90)
    pos = torch.randint(0, L, (L, len(dims)), generator=g, device=DEV, dtype=torch.int32)
    angles = torch.cat([pos[:, a:a + 1].double() * torch.tensor(10000.0 ** (-2.0 * np.arange(d // 2) / d), device=DEV) for a, d in enumerate(dims)], dim=1)
    q = torch.randn((1, L, H, D), generator=g, device=DEV).to(dtype)
    w = torch.linspace(0.5, 2.0, D, device=DEV)
    P = sum(dims) // 2

    def within(got, ref, size, kind):
        assert float(((got.double() - ref).abs() - (HALF_ULP[kind] * ref.abs() + 32 * U * size)).max()) <= 0.0

    y, _ = oq.qk_norm_rope(plan, q, None, pos, w, eps=EPS, out_dtype=out)
    x64, w64 = q.double(), w.double()
    r = torch.rsqrt(x64.square().mean(-1, keepdim=True) + EPS)
    n = x64 * r * w64
    within(y, _turned(n, angles, halves), _device_pair_length(n, P, halves), out)
    if dtype == out:
        within(oq.axial_rope(plan, q, pos, inverse=True), _turned(x64, angles, halves, -1.0), _device_pair_length(x64, P, halves), dtype)
    del y, n
    dy = torch.randn((1, L, H, D), generator=g, device=DEV).to(out)
    gq, _, dw, _ = oq.qk_norm_rope_backward(plan, dy, None, q, None, pos, w, eps=EPS)
    t = _turned(dy.double(), angles, halves, -1.0)
    dot = (t * w64 * x64).mean(-1, keepdim=True)
    length = _device_pair_length(t, P, halves) * w64
    within(gq, r * (t * w64 - x64 * r * r * dot), r * (length + x64.abs() * r * r * (length * x64.abs()).mean(-1, keepdim=True)), dtype)
    terms = (_device_pair_length(t, P, halves) * x64.abs() * r).sum((0, 1, 2))
    assert ((dw.double() - (t * x64 * r).sum((0, 1, 2))).abs() <= (10 * (L * H) ** 0.5 + 32) * U * terms).all()


def test_more_waves_than_a_launch_holds():
    # heads of 264 values take a wave each: 2^26 of them and a few more, from one row of each of 40 positions
    L, D = 2 ** 26 + 5, 264
    plan = oq.rope_plan((264,), (40,))
    x = _rows((1, 1, 1, D), BF16, 95)
    pos = (torch.arange(L, device=DEV) % 40).to(torch.int32)[:, None]
    w = torch.linspace(0.5, 2.0, D, device=DEV)
    few = x.expand(1, 40, 1, D)
    out = torch.empty((1, L, 1, D), dtype=BF16, device=DEV)
    for call in (lambda x, p, y: oq.axial_rope(plan, x, p, out=y), lambda x, p, y: oq.qk_norm_rope(plan, x, None, p, w, eps=EPS, q_out=y)[0]):
        want = call(few, pos[:40].contiguous(), None)[0]
        out.zero_()
        call(x.expand(1, L, 1, D), pos, out)
        for at in range(0, L, 40 << 16):
            got = out[0, at:at + (40 << 16)]
            assert torch.equal(got, want.repeat((got.shape[0] + 39) // 40, 1, 1)[:got.shape[0]])


def _instances(call):
    """(kernel, layout, non-temporal, rows in flight or None, grid) of each rotation that the call launches, off its mangled name."""
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(launches_module, "short_name", str)
        found = [(re.search(r"\d\d((?:axial|qk)_\w*?kernel)I.*?Li(\d)ELb([01])E(?:Li(\d)E)?EEvNS", r.kernel), r.grid) for r in launches_module.launches(call)]
    return [(m[1], int(m[2]), m[3] == "1", m[4] and int(m[4]), grid) for m, grid in found if m]


@pytest.mark.parametrize("D,dims,layout,streams", [(80, (40, 40), "dense", True), (80, (40, 40), "padded", True), (80, (40, 40), "heads", False),
                                                   (128, (64, 64), "heads", True), (160, (64, 64), "dense", False)])
def test_non_temporal_accesses_go_by_what_lies_together(D, dims, layout, streams):
    # above 160 MiB in and out; heads of 80 values are no whole lines, 24 of a token are; nor are 9 heads of 160
    H = 9 if D == 160 else 24
    L = (170 << 20) // (H * D * 4) + 1
    plan, pos, _ = _plan_and_positions(dims, 1, L, 96, False)
    q, dq = _rows((1, L, H, D), BF16, 97), _rows((1, L, H, D), BF16, 98)
    want = oq.qk_norm_rope(plan, q, None, pos)[0], oq.qk_norm_rope_backward(plan, dq, None, q, None, pos)[0]

    def lay(t):
        if layout == "heads":
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        return torch.nn.functional.pad(t, (8, 0))[..., 8:] if layout == "padded" else t

    q, dq, y = lay(q), lay(dq), lay(torch.zeros_like(q))
    forward = lambda: oq.qk_norm_rope(plan, q, None, pos, q_out=y)  # noqa: E731
    backward = lambda: oq.qk_norm_rope_backward(plan, dq, None, q, None, pos, q_grad=y)  # noqa: E731
    for call, ref, name in ((forward, want[0], "axial_rope_kernel"), (backward, want[1], "qk_norm_rope_backward_kernel")):
        call()
        assert torch.equal(y, ref)
        (kernel, _, non_temporal, _, _), = _instances(call)
        assert kernel == name and non_temporal == streams


# --- several rows to a wave and several waves to a token -------------------------------------------
@pytest.mark.parametrize("Hq,Hk,chunks,rows", [(24, 8, 1, 6), (40, 24, 2, 6), (43, 13, 2, 6), (16, 5, 1, 3)])
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_heads_of_many_tokens(Hq, Hk, chunks, rows, large, halves, dtype):
    # heads of 128 are four to a wave side by side: 43 are two waves of 6 and 5 rows, whose last one has 3 heads
    D, dims = 128, (16, 56, 40)
    L = (161 << 20) // ((Hq + Hk) * D * 4) if large else 1103    # above 160 MiB the accesses are non-temporal
    plan, pos, angles = _plan_and_positions(dims, 1, L, 100, halves)
    angles, P = torch.tensor(angles[0], device=DEV), sum(dims) // 2
    g = torch.Generator(device=DEV).manual_seed(101)
    q, k, dq, dk = (torch.randn((1, L, h, D), generator=g, device=DEV).to(t) for h, t in ((Hq, dtype), (Hk, dtype), (Hq, BF16), (Hk, BF16)))
    wq, wk = torch.linspace(0.5, 2.0, D, device=DEV), torch.linspace(2.0, 0.5, D, device=DEV)
    forward = lambda: oq.qk_norm_rope(plan, q, k, pos, wq, wk, eps=EPS, out_dtype=BF16)  # noqa: E731
    backward = lambda: oq.qk_norm_rope_backward(plan, dq, dk, q, k, pos, wq, wk, eps=EPS)  # noqa: E731
    (_, _, non_temporal, _, grid), = _instances(forward)
    # (a half of the turned part, 56 values of bf16, is no whole line)
    assert non_temporal == (large and not halves) and grid == ((L * chunks + 3) // 4, 2, 1)
    (_, _, non_temporal, in_flight, _), = _instances(backward)
    assert non_temporal == (L * (Hq + Hk) * D * (2 * q.element_size() + 2) > 160 << 20 and not halves) and in_flight == rows

    def within(name, got, ref, size, kind):
        over = float(((got.double() - ref).abs() - (HALF_ULP[kind] * ref.abs() + 32 * U * size)).max())
        assert over <= 0.0, f"{name}: {over} beyond its bar"

    got, grads = forward(), backward()
    for i, (name, x, dy, w) in enumerate((("q", q, dq, wq), ("k", k, dk, wk))):
        x, w = x.double(), w.double()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = x * r * w
        within(name, got[i], _turned(n, angles, halves), _device_pair_length(n, P, halves), BF16)
        t = _turned(dy.double(), angles, halves, -1.0)
        length = _device_pair_length(t, P, halves)
        ref = r * (t * w - x * r * r * (t * w * x).mean(-1, keepdim=True))
        size = r * (length * w + x.abs() * r * r * (length * w * x.abs()).mean(-1, keepdim=True))
        within(f"{name} grad", grads[i], ref, size, dtype)
        terms = (length * x.abs() * r).sum((0, 1, 2))
        bar = (10 * (L * x.shape[2]) ** 0.5 + 32) * U * terms
        assert ((grads[2 + i].double() - (t * x * r).sum((0, 1, 2))).abs() <= bar).all(), f"{name} weight grad"
