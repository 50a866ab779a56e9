"""GPU parity of the layer norms and their gradients against the fp64 oracle, at the sizes, layouts and values where they can
go wrong.

Bars, per value, with u = 2^-24.  A mean of N <= 12288 values is a sum of at most 24 in a row, then pairwise over lanes and
waves: it is off by at most 40 u mean|x|, so a unit n = (x - mean) r is off by 64 u U with U = r (|x| + mean|x|) (the rest: the
difference, r, whose sum of squares is of deviations, and the product).  y = n g + b then is off by half an ulp of its type and
64 u (U |g| + |b|).  dx = r (h - mean h - n mean(h n)), h = dy g: 64 u r (|h| + mean|h| + 2 U mean(|h| U)).  A gradient of the
weights is a sum of M terms: (10 sqrt(M) + 64) u sum|dy| U (Higham and Mary, SIAM J. Sci. Comput. 2019, lambda = 10), the bias's
the same with 1 for U.
"""

import numpy as np
import pytest
import torch

import oracle
import paper_2607_02461_amd as oq
from paper_2607_02461_amd.launches import launches

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: U}
EPS = 1e-6


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _within(name, got, ref, bar):
    got = _f64(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    over = np.abs(got - ref) / np.maximum(bar, 1e-300)
    assert got.size == 0 or over.max() <= 1.0, f"{name}: {over.max():.3f} of the bar at {np.unravel_index(over.argmax(), over.shape)}"


def _rows(B, L, N, dtype, seed, layout="dense", place=0.5):
    """Rows with channels of different size and place, in one of the layouts they have in use."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, N), generator=g) * torch.exp(0.5 * torch.randn((N,), generator=g)) + place * torch.randn((N,), generator=g)
    x = x.to(dtype).to(DEV)
    if layout == "apart":        # rows of N + 5 values, so that they begin anywhere
        whole = torch.full((B, L, N + 5), float("nan"), dtype=dtype, device=DEV)
        whole[..., 3:N + 3] = x
        return whole[..., 3:N + 3]
    if layout == "tokens":       # [L, B, N] in memory
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    return x


def _weights(B, N, dtype, seed, modulate):
    g = torch.Generator().manual_seed(seed)
    if modulate:                 # two of the six parts of the modulation projection's output
        return (0.5 * torch.randn((B, 6 * N), generator=g)).to(dtype).to(DEV).chunk(6, dim=-1)[1:3]
    return tuple((k + 0.5 * torch.randn((N,), generator=g)).to(dtype).to(DEV) for k in (1, 0))


def _gain(w, modulate):
    return (1 + _f64(w))[:, None] if modulate else _f64(w)


def _check(x, w, b, modulate, y, dy=None, grads=None, eps=EPS):
    x64 = _f64(x)
    gain = 1.0 if w is None else _gain(w, modulate)
    shift = 0.0 if b is None else (_f64(b)[:, None] if modulate else _f64(b))
    r = 1 / np.sqrt(x64.var(-1, keepdims=True) + eps)
    unit = r * (np.abs(x64) + np.abs(x64).mean(-1, keepdims=True))
    ref = oracle.layer_norm(x64, gain, shift, eps)
    _within("y", y, ref, HALF[y.dtype] * np.abs(ref) + 64 * U * (unit * np.abs(gain) + np.abs(shift)))
    if grads is None:
        return
    dy64, over = _f64(dy), 1 if modulate else (0, 1)
    dx, dw, db = oracle.layer_norm_backward(dy64, x64, gain, eps)
    h = np.abs(dy64 * gain)
    size = r * (h + h.mean(-1, keepdims=True) + 2 * unit * (h * unit).mean(-1, keepdims=True))
    _within("dx", grads[0], dx, HALF[grads[0].dtype] * np.abs(dx) + 64 * U * size)
    rows = x64.shape[1] if modulate else x64.shape[0] * x64.shape[1]
    grow = (10 * rows ** 0.5 + 64) * U
    _within("dw", grads[1], dw.sum(over), grow * (np.abs(dy64) * unit).sum(over) + U * np.abs(dw.sum(over)))
    _within("db", grads[2], db.sum(over), grow * np.abs(dy64).sum(over) + U * np.abs(db.sum(over)))


# one row to many, widths of one value, within a piece, of a piece's and a wave's edge, odd ones, of every number of pieces
SHAPES = [(1, 1, 1), (1, 3, 7), (2, 5, 8), (1, 2, 63), (3, 4, 512), (1, 9, 513), (2, 3, 1999), (1, 1, 5120), (2, 700, 192), (1, 1100, 260), (1, 513, 1536),
          (4, 300, 769), (1, 600, 3071), (2, 2, 12288), (1, 600, 12288), (1, 515, 6151), (1, 520, 5120)]


@pytest.mark.parametrize("B,L,N", SHAPES)
@pytest.mark.parametrize("modulate", [False, True])
@pytest.mark.parametrize("dtype,out,weights,layout", [(BF16, BF16, F32, "dense"), (F32, BF16, F32, "apart"), (F32, F32, BF16, "dense"),
                                                      (BF16, F32, BF16, "tokens"), (BF16, BF16, BF16, "apart")])
def test_norms_and_gradients(B, L, N, modulate, dtype, out, weights, layout):
    x, (w, b) = _rows(B, L, N, dtype, 1, layout), _weights(B, N, weights, 2, modulate)
    dy = _rows(B, L, N, out, 3, layout)
    forward, backward = (oq.layer_norm_modulate, oq.layer_norm_modulate_backward) if modulate else (oq.layer_norm, oq.layer_norm_backward)
    y = forward(x, w, b, eps=EPS, out_dtype=out)
    assert y.dtype == out and y.shape == x.shape
    grads = backward(dy, x, w, eps=EPS)
    assert grads[0].dtype == dtype and grads[1].dtype == grads[2].dtype == F32 and grads[1].shape == ((B, N) if modulate else (N,))
    _check(x, w, b, modulate, y, dy, grads)


def test_without_weights_and_tokens_of_one_batch():
    x, dy = _rows(1, 37, 640, BF16, 4)[0], _rows(1, 37, 640, BF16, 5)[0]
    one = torch.ones((640,), device=DEV)
    assert torch.equal(oq.layer_norm(x), oq.layer_norm(x, one, torch.zeros_like(one)))
    assert torch.equal(oq.layer_norm_modulate(x, None, None), oq.layer_norm(x))
    got, want = oq.layer_norm_backward(dy, x), oq.layer_norm_backward(dy, x, one)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    scale = 0.5 * torch.randn((1, 640), device=DEV)
    got = oq.layer_norm_modulate_backward(dy, x, scale)
    want = oq.layer_norm_backward(dy, x, 1 + scale[0])
    assert all(torch.equal(a.flatten(), b.flatten()) for a, b in zip(got, want))
    bias = torch.randn((640,), device=DEV)
    _check(x[None], None, bias, False, oq.layer_norm(x, None, bias, out_dtype=F32)[None])


@pytest.mark.parametrize("N", [100, 5120])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_means_far_from_zero(N, dtype):
    # a mean 10^4 deviations away: squares of the values lose the variance, squares of deviations do not
    g = torch.Generator().manual_seed(6)
    x = (1e4 + torch.randn((1, 5, N), generator=g)).to(F32) if dtype == F32 else (256 + torch.randint(0, 3, (1, 5, N), generator=g) * 2).to(BF16)
    x = x.to(DEV)
    _check(x, None, None, False, oq.layer_norm(x, out_dtype=F32), _rows(1, 5, N, F32, 7), oq.layer_norm_backward(_rows(1, 5, N, F32, 7), x))


@pytest.mark.parametrize("N", [257, 1025, 1538, 2049])
@pytest.mark.parametrize("rows", [8, 700])
def test_last_values_alone_in_their_wave(N, rows):
    # the row's last values, a piece that its end cuts, are another wave's than the values before them, and far from them: 10^6
    # times their size.  Each wave writes its own values alone: the others', by deviations from its own mean, would be off by
    # half an ulp of 10^6, up to N / 128 times the bar
    x = _rows(1, rows, N, F32, 31)
    x[..., N // 4 * 4:] = 1e6
    dy = _rows(1, rows, N, F32, 32)
    y, grads = oq.layer_norm(x), oq.layer_norm_backward(dy, x)
    _check(x, None, None, False, y, dy, grads)
    assert torch.equal(oq.layer_norm(x), y) and torch.equal(oq.layer_norm_backward(dy, x)[0], grads[0])


@pytest.mark.parametrize("N", [300, 1999, 5120, 12288])
@pytest.mark.parametrize("rows", [3, 700])
@pytest.mark.parametrize("dtype,spread", [(F32, 0.0), (F32, 1e-3), (BF16, None)])
def test_rows_that_vary_by_less_than_their_means_rounding(N, rows, dtype, spread):
    """A wave's mean is a quotient off by at most 40 u |x| and the mean of the deviations from it, which are exact (values within
    a factor of two of the quotient) and themselves up to 40 u |x| beside a row's own; their mean is off by 41 u of that.  The waves'
    means meet as differences of up to 80 u |x|, off by (16 + 4) u of what is summed, and the row's by as much: D = 2^13 u^2 |x| in
    all.  A unit is off by r D, and by 64 u of itself: r, whose squares are of deviations."""
    g = torch.Generator().manual_seed(41)
    place = torch.linspace(1000.1, 3333.3, rows)[:, None]
    if spread is None:                            # one value a few of its steps from the others
        x = place.expand(rows, N).clone()
        x[:, N // 3] *= 1.03125
    else:
        x = place + spread * torch.randn((rows, N), generator=g)
    x = x.to(dtype)[None].to(DEV)
    (w, b), dy = _weights(1, N, F32, 42, False), _rows(1, rows, N, F32, 43)
    y, (dx, dw, db) = oq.layer_norm(x, w, b, out_dtype=F32), oq.layer_norm_backward(dy, x, w)
    x64, dy64, gain, shift = _f64(x), _f64(dy), _f64(w), _f64(b)
    x64 = x64 - x64[..., :1]                      # exact: the same deviations, without the oracle's own rounding of the mean
    r = 1 / np.sqrt(x64.var(-1, keepdims=True) + EPS)
    off = r * 2.0 ** 13 * U * U * 3400.0
    unit = r * np.abs(x64 - x64.mean(-1, keepdims=True))
    ref = oracle.layer_norm(x64, gain, shift, EPS)
    _within("y", y, ref, U * np.abs(ref) + (64 * U * unit + off) * np.abs(gain) + 2 * U * np.abs(shift))
    want, gains, shifts = oracle.layer_norm_backward(dy64, x64, gain, EPS)
    h = np.abs(dy64 * gain)
    most = unit + off
    mean_hn = (h * most).mean(-1, keepdims=True)
    size = r * (64 * U * (h + h.mean(-1, keepdims=True) + 2 * most * mean_hn) + off * (mean_hn + most * h.mean(-1, keepdims=True)))
    _within("dx", dx, want, HALF[dtype] * np.abs(want) + size)
    grow = (10 * rows ** 0.5 + 64) * U
    _within("dw", dw, gains.sum((0, 1)), grow * (np.abs(dy64) * unit).sum((0, 1)) + 1.01 * (np.abs(dy64) * off).sum((0, 1)))
    _within("db", db, shifts.sum((0, 1)), grow * np.abs(dy64).sum((0, 1)))


def test_rows_without_variance_and_values_that_are_not_finite():
    x = _rows(1, 8, 300, F32, 8)
    x[0, 1], x[0, 2], x[0, 4, 7], x[0, 6, 299] = 0.0, 3.0, float("nan"), float("inf")
    w, b = _weights(1, 300, F32, 9, False)
    y = oq.layer_norm(x, w, b, out_dtype=F32)
    assert torch.equal(y[0, 1], b) and torch.equal(y[0, 2], b)
    bad = torch.zeros(8, dtype=torch.bool, device=DEV)
    bad[4] = bad[6] = True
    assert torch.isfinite(y[0, ~bad]).all() and not torch.isfinite(y[0, bad]).any()
    dx, _, _ = oq.layer_norm_backward(_rows(1, 8, 300, F32, 10), x, w)
    assert torch.isfinite(dx[0, ~bad]).all() and not torch.isfinite(dx[0, bad]).any()
    big = torch.full((1, 2, 300), 1e30, device=DEV)
    big[0, :, ::2] = -1e30
    assert torch.equal(oq.layer_norm(big, w, b, out_dtype=F32)[0, 0], b)   # the variance passes fp32: the bias


@pytest.mark.parametrize("modulate", [False, True])
def test_in_place_broadcast_inputs_and_rows_beside_the_outputs(modulate):
    x, (w, b) = _rows(3, 70, 264, BF16, 11), _weights(3, 264, F32, 12, modulate)
    dy = _rows(3, 70, 264, BF16, 13)
    forward, backward = (oq.layer_norm_modulate, oq.layer_norm_modulate_backward) if modulate else (oq.layer_norm, oq.layer_norm_backward)
    want, grads = forward(x, w, b), backward(dy, x, w)
    whole = torch.full((3, 71, 270), 7.0, dtype=BF16, device=DEV)
    out = whole[:, :70, 2:266]
    assert forward(x, w, b, out=out) is out and torch.equal(out, want)
    out.fill_(7.0)
    assert (whole == 7.0).all()
    for place in ("x", "dy"):
        a, c = x.clone(), dy.clone()
        got = backward(c, a, w, x_grad=a if place == "x" else c)
        assert all(torch.equal(s, t) for s, t in zip(got, grads))
    y = x.clone()
    forward(y, w, b, out=y)
    assert torch.equal(y, want)
    # one row for all tokens, one batch for all: the gradients count each of them
    row = x[:1, :1].expand(3, 70, 264)
    assert torch.equal(forward(row, w, b), forward(row.contiguous(), w, b))
    got, want = backward(dy, row, w), backward(dy, row.contiguous(), w)
    assert all(torch.equal(s, t) for s, t in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [300, 1999, 5120])
@pytest.mark.parametrize("size", [2.0 ** 66, 2.0 ** 100])
def test_rows_whose_variance_passes_fp32(dtype, N, size):
    # r is 0: the bias, and no gradient but the bias's
    x = _rows(1, 5, N, dtype, 71) * size
    (w, b), dy = _weights(1, N, F32, 72, False), _rows(1, 5, N, F32, 73)
    assert torch.equal(oq.layer_norm(x, w, b, out_dtype=F32), b.expand(1, 5, N))
    dx, dw, db = oq.layer_norm_backward(dy, x, w)
    assert not dx.any() and not dw.any()
    _within("db", db, _f64(dy).sum((0, 1)), (10 * 5 ** 0.5 + 64) * U * np.abs(_f64(dy)).sum((0, 1)))


@pytest.mark.parametrize("modulate", [False, True])
@pytest.mark.parametrize("N", [63, 640])
def test_gradients_against_differences(N, modulate):
    # fp32 throughout: each gradient is within 256 u of its terms' size, and a central difference of step s within s^2 of the third
    # derivative: 1e-4 in fp64 leaves some 1e-8 of a loss of that size, and its rounding 1e-16 / 1e-4
    x, (w, b), dy = _rows(2, 9, N, F32, 61), _weights(2, N, F32, 62, modulate), _rows(2, 9, N, F32, 63)
    forward, backward = (oq.layer_norm_modulate, oq.layer_norm_modulate_backward) if modulate else (oq.layer_norm, oq.layer_norm_backward)
    grads = [_f64(t) for t in backward(dy, x, w)]
    r = np.random.default_rng(3)
    values = [_f64(t) for t in (x, w, b)]
    along = [r.standard_normal(t.shape) for t in values]

    def loss(step):
        x, w, b = (t + step * d for t, d in zip(values, along))
        return float((oracle.layer_norm(x, *((1 + w[:, None], b[:, None]) if modulate else (w, b))) * _f64(dy)).sum())

    want = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = sum(float((g * d).sum()) for g, d in zip(grads, along))
    size = np.sqrt(sum(float(((g * d) ** 2).sum()) for g, d in zip(grads, along)))
    terms = sum(float(np.abs(g * d).sum()) for g, d in zip(grads, along))
    assert abs(got - want) <= 1e-6 * size + 256 * U * terms, (got, want, size)
    assert forward(x, w, b).dtype == F32


@pytest.mark.parametrize("rows,step", [(37, 1), (200, 1), (37, 3)])
def test_rows_that_are_windows_of_a_signal(rows, step):
    # windows of 64 values that lie `step` apart
    signal = _rows(2, 1, (rows - 1) * step + 64, BF16, 51)[:, 0]
    for x in (signal[0].unfold(0, 64, step), signal.unfold(1, 64, step)):
        assert x.shape[-2:] == (rows, 64) and x.stride()[-2:] == (step, 1)
        dy = _rows(1, rows, 64, BF16, 52)[0].expand(x.shape)
        assert torch.equal(oq.layer_norm(x), oq.layer_norm(x.contiguous()))
        assert all(torch.equal(a, b) for a, b in zip(oq.layer_norm_backward(dy, x), oq.layer_norm_backward(dy, x.contiguous())))


def test_one_scale_for_each_token_of_many():
    # batches of one row each, more of them than a grid's second dimension holds
    B, N = 70000, 24
    x, (scale, shift) = _rows(B, 1, N, BF16, 14), _weights(B, N, F32, 15, True)
    dy = _rows(B, 1, N, BF16, 16)
    _check(x, scale, shift, True, oq.layer_norm_modulate(x, scale, shift), dy, oq.layer_norm_modulate_backward(dy, x, scale))


def test_no_rows():
    for B, L in ((0, 5), (2, 0)):
        x = torch.empty((B, L, 16), dtype=BF16, device=DEV)
        assert oq.layer_norm(x).shape == x.shape
        dx, dw, db = oq.layer_norm_backward(x, x)
        assert dx.shape == x.shape and not dw.any() and not db.any() and dw.shape == (16,)
        dx, dw, db = oq.layer_norm_modulate_backward(x, x, torch.zeros((B, 16), device=DEV))
        assert dw.shape == (B, 16) and not dw.any() and not db.any()


def test_rows_beyond_32_bit_offsets():
    B, L, N = 1, 210_000, 12288   # 2.6e9 values
    x = torch.empty((B, L, N), dtype=BF16, device=DEV)
    for at in range(0, L, 30_000):
        x[0, at:at + 30_000].normal_(1.0, 2.0)
    y = oq.layer_norm(x)
    dx, dw, db = oq.layer_norm_backward(y, x)
    rows = [0, 1, 174_762, 174_763, L - 1]
    _check(x[:, rows], None, None, False, y[:, rows])
    ref, _, _ = oracle.layer_norm_backward(_f64(y[:, rows]), _f64(x[:, rows]))
    unit = np.abs(_f64(x[:, rows])) + np.abs(_f64(x[:, rows])).mean(-1, keepdims=True)
    h = np.abs(_f64(y[:, rows]))
    r = 1 / np.sqrt(_f64(x[:, rows]).var(-1, keepdims=True) + EPS)
    size = r * (h + h.mean(-1, keepdims=True) + 2 * r * unit * (h * r * unit).mean(-1, keepdims=True))
    _within("dx", dx[:, rows], ref, HALF[BF16] * np.abs(ref) + 64 * U * size)
    total = torch.zeros((N,), dtype=torch.float64, device=DEV)
    for at in range(0, L, 30_000):
        total += y[0, at:at + 30_000].double().sum(0)
    assert float((db - total).abs().max()) <= (10 * L ** 0.5 + 64) * U * 4.0 * L   # |y| below 4 on average, by far


def test_streams_and_graphs():
    x, (w, b) = _rows(2, 600, 640, BF16, 17), _weights(2, 640, F32, 18, True)
    dy = _rows(2, 600, 640, BF16, 19)

    def both():
        return (oq.layer_norm_modulate(x, w, b),) + tuple(oq.layer_norm_modulate_backward(dy, x, w))

    want = both()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(both())
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for g in got for a, c in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for seed in range(3):
        x.copy_(_rows(2, 600, 640, BF16, 20 + seed))
        dy.copy_(_rows(2, 600, 640, BF16, 30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(held, both()))
    assert len(launches(lambda: oq.layer_norm_modulate(x, w, b, out=held[0]))) == 1


def test_refusals():
    x = torch.zeros((2, 3, 16), dtype=BF16, device=DEV)
    w = torch.ones((16,), device=DEV)
    for call, word in ((lambda: oq.layer_norm(x.cpu()), "GPU"), (lambda: oq.layer_norm(x.half()), "bf16 or fp32"), (lambda: oq.layer_norm(x[0, 0]), "token"),
                       (lambda: oq.layer_norm(x[..., ::2]), "contiguous"), (lambda: oq.layer_norm(x, w[:8]), "shape"), (lambda: oq.layer_norm(x, w, w.to(BF16)), "one type"),
                       (lambda: oq.layer_norm(x, w.cpu()), "shape"), (lambda: oq.layer_norm(x, out_dtype=torch.float16), "out_dtype"),
                       (lambda: oq.layer_norm(x, out=x[:1].expand(2, 3, 16)), "overlap"), (lambda: oq.layer_norm(x, out=x[:, :2]), "shape"),
                       (lambda: oq.layer_norm_modulate(x, w, w), "shape"), (lambda: oq.layer_norm_modulate(x, w.expand(3, 16), None), "shape"),
                       (lambda: oq.layer_norm_backward(x[:1], x), "shape"), (lambda: oq.layer_norm_backward(x, x, x_grad=x.float()), "must be")):
        with pytest.raises(ValueError, match=word):
            call()
    for call in (lambda: oq.layer_norm(x, eps=-1.0), lambda: oq.layer_norm(torch.zeros((1, 12289), device=DEV))):
        with pytest.raises(oq.OrbitError):
            call()
