"""GPU parity of the low-rank adapters against the fp64 oracle.

Bars, per value, with u = 2^-24.  h = x A^T is an fp32 sum of K exact products: within 10 sqrt(K) u |x| |A| (Higham and
Mary, SIAM J. Sci. Comput. 2019, lambda = 10; |x| |A| the product of the absolute values).  h enters the second product
as two bf16 values, within 2^-16 of it, and r terms add up in fp32: so with P = scale |h bar| |B| and
H = scale (|x| |A|) |B|, |y - ref| <= half an ulp of y's type + 2^-16 P + 10 (sqrt(K) + sqrt(r + 1)) u H + 2 u |base|.
P <= H, and sqrt(r + 1) <= 12: the bar is ulp |ref| + (2^-16 + (10 sqrt(K) + 120) u) H + 2 u |base|.  The same holds for
dx with N for K.  A gradient adds up n rows of such values: ulp of fp32 + (2^-16 + (10 sqrt(K or N) + 10 sqrt(n) + 120) u) H,
H again the products of absolute values.
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
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, F32 = torch.bfloat16, torch.float32


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _randn(shape, seed, scale=1.0, dtype=BF16):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).to(DEV)


class Batch:
    def __init__(self, M, K, N, R, starts, adapters, ranks, scales, dtype=BF16, seed=1):
        self.lists = dict(starts=starts, adapters=adapters, ranks=ranks, scales=scales)
        self.M, self.K, self.N, self.R, self.n, self.dtype = M, K, N, R, len(ranks), dtype
        self.plan = oq.lora_plan(M, **self.lists)
        self.x, self.base, self.dy = _randn((M, K), seed), _randn((M, N), seed + 1, 1.0, dtype), _randn((M, N), seed + 2, 0.1)
        # what lies beyond an adapter's rank is not a number, and does not matter
        self.A, self.B = _randn((self.n, R, K), seed + 3, K ** -0.5), _randn((self.n, N, R), seed + 4, 0.3)
        for a, r in enumerate(ranks):
            self.A[a, r:] = float("nan")
            self.B[a, :, r:] = float("nan")
        self.h = torch.full((M, R), float("nan"), dtype=F32, device=DEV)

    def numbers(self, absolute=False):
        got = [np.nan_to_num(_f64(t)) for t in (self.x, self.A, self.B)]
        return [np.abs(v) for v in got] if absolute else got

    def check_forward(self, y, name="y"):
        x, A, B = self.numbers()
        base = _f64(self.base)
        ref = oracle.lora_add(x, A, B, base, **self.lists)
        size = oracle.lora_add(*self.numbers(True), np.zeros_like(base), **self._positive())
        bar = HALF_ULP[self.dtype] * np.abs(ref) + (2.0 ** -16 + (10 * np.sqrt(self.K) + 120) * U) * size + 2 * U * np.abs(base)
        _within(name, _f64(y), ref, bar)

    def check_h(self, h):
        x, A, _ = self.numbers()
        ref, size = np.zeros((self.M, self.R)), np.zeros((self.M, self.R))
        starts, M = self.lists["starts"], self.M
        for first, end, a in zip(starts, list(starts[1:]) + [M], self.lists["adapters"]):
            if a >= 0:
                r = self.lists["ranks"][a]
                ref[first:end, :r] = x[first:end] @ A[a, :r].T
                size[first:end, :r] = np.abs(x[first:end]) @ np.abs(A[a, :r].T)
        _within("h", _f64(h), ref, (10 * np.sqrt(self.K) + 2) * U * size)

    def _positive(self):
        return self.lists | dict(scales=[abs(s) for s in self.lists["scales"]])

    def check_backward(self, dx, dA, dB, base=None):
        x, A, B = self.numbers()
        dy = _f64(self.dy)
        refs = list(oracle.lora_add_backward(dy, x, A, B, **self.lists))
        sizes = oracle.lora_add_backward(np.abs(dy), *self.numbers(True), **self._positive())
        slack = 0.0
        if base is not None:
            refs[0] = refs[0] + _f64(base)
            slack = 2 * U * np.abs(_f64(base))
        assert dx.dtype == BF16 and dA.dtype == F32 and dB.dtype == F32
        grow = 10 * np.sqrt(max(self.K, self.N)) + 120
        _within("dx", _f64(dx), refs[0], HALF_ULP[BF16] * np.abs(refs[0]) + (2.0 ** -16 + grow * U) * sizes[0] + slack)
        grow += 10 * np.sqrt(self.M)
        for name, got, ref, size in (("dA", dA, refs[1], sizes[1]), ("dB", dB, refs[2], sizes[2])):
            _within(name, _f64(got), ref, U * np.abs(ref) + (2.0 ** -16 + grow * U) * size)

    def forward(self, **kw):
        return oq.lora_add(self.plan, self.x, self.A, self.B, self.base, h=self.h, **kw)

    def backward(self, **kw):
        return oq.lora_add_backward(self.plan, self.dy, self.x, self.A, self.B, self.h, **kw)


def _within(name, got, ref, bar):
    assert np.isfinite(got).all(), f"{name}: not finite"
    over = np.abs(got - ref) / np.maximum(bar, 1e-300)
    assert got.size == 0 or over.max() <= 1.0, f"{name}: {over.max():.3f} of the bar at {np.unravel_index(over.argmax(), over.shape)}"


BATCHES = {
    "one row": dict(M=1, starts=[0], adapters=[0], ranks=[8], scales=[1.0]),
    "rows of their own": dict(M=5, starts=[0, 1, 2, 3, 4], adapters=[3, 0, -1, 2, 1], ranks=[8, 3, 1, 5], scales=[1.0, -0.5, 2.0, 0.25]),
    "ragged": dict(M=333, starts=[0, 17, 17, 81, 82, 200], adapters=[1, 0, 2, -1, 0, 1], ranks=[8, 7, 2], scales=[1.0, 0.5, -2.0]),
    "late start": dict(M=70, starts=[66], adapters=[0], ranks=[4], scales=[3.0]),
    "tile edges": dict(M=257, starts=[0, 64, 128, 129, 193], adapters=[0, 1, 0, 1, 0], ranks=[8, 6], scales=[1.0, 1.0]),
    "nobody": dict(M=40, starts=[0], adapters=[-1], ranks=[8, 8], scales=[1.0, 1.0]),
    "no segments": dict(M=9, starts=[], adapters=[], ranks=[8], scales=[1.0]),
    "rank zero": dict(M=30, starts=[0, 10], adapters=[0, 1], ranks=[0, 8], scales=[1.0, 1.0]),
    "long": dict(M=2500, starts=[0, 1200], adapters=[0, 1], ranks=[8, 8], scales=[0.5, 1.0]),
}


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("K,N", [(8, 1), (40, 64), (512, 333), (1032, 770), (3072, 520)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_batches(name, K, N, dtype):
    b = Batch(K=K, N=N, R=8, dtype=dtype, **BATCHES[name])
    y = b.forward()
    assert y.dtype == dtype
    b.check_forward(y)
    b.check_h(b.h)
    b.check_backward(*b.backward())


@pytest.mark.parametrize("R,ranks", [(8, [8, 1]), (16, [16, 9]), (24, [17, 24]), (32, [32, 31]), (40, [33, 40]), (64, [64, 50]), (72, [65, 3]),
                                     (96, [96, 70]), (128, [128, 127])])
@pytest.mark.parametrize("K,N", [(72, 200), (1024, 515)])
def test_ranks(R, ranks, K, N):
    b = Batch(150, K, N, R, [0, 33, 100], [0, 1, 0], ranks, [0.5, 2.0])
    b.check_forward(b.forward())
    b.check_h(b.h)
    b.check_backward(*b.backward())


@pytest.mark.parametrize("N", [1, 2, 7, 9, 63, 65, 127, 129, 255, 257])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_odd_widths_leave_what_is_beside_them(N, dtype):
    M, K, R = 37, 200, 16
    b = Batch(M, K, N, R, [0, 20], [0, 1], [16, 5], [1.0, 0.5], dtype)
    whole = torch.full((M + 2, N + 5), 7.0, dtype=dtype, device=DEV)
    y = whole[1:-1, 3:3 + N]                     # rows of odd stride that begin at odd elements
    b.check_forward(b.forward(out=y))
    assert (whole[0] == 7).all() and (whole[-1] == 7).all() and (whole[:, :3] == 7).all() and (whole[:, 3 + N:] == 7).all()
    # the same for inputs: their surroundings are not numbers
    plain = b.backward()
    for field in ("x", "dy"):
        t = getattr(b, field)
        whole = torch.full((M + 2, t.shape[1] + 7), float("nan"), dtype=BF16, device=DEV)
        whole[1:-1, 5:5 + t.shape[1]] = t
        setattr(b, field, whole[1:-1, 5:5 + t.shape[1]])
    b.check_forward(b.forward())
    assert all(torch.equal(p, q) for p, q in zip(plain, b.backward()))
    whole = torch.full((M + 2, K + 3), 7.0, dtype=BF16, device=DEV)
    dx = whole[1:-1, 1:1 + K]
    b.check_backward(*b.backward(out=dx))
    assert (whole[0] == 7).all() and (whole[-1] == 7).all() and (whole[:, :1] == 7).all() and (whole[:, 1 + K:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_added_gradient(dtype):
    b = Batch(130, 264, 77, 8, [0, 50, 90], [0, -1, 1], [8, 4], [1.0, 2.0], dtype)
    want = b.forward()
    y = b.base.clone()
    assert oq.lora_add(b.plan, b.x, b.A, b.B, y, out=y).data_ptr() == y.data_ptr() and torch.equal(y, want)
    from_projection = _randn((130, 264), 9)
    dx, dA, dB = b.backward(base=from_projection)
    b.check_backward(dx, dA, dB, from_projection)
    held = from_projection.clone()
    got = b.backward(base=held, out=held)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dA) and torch.equal(got[2], dB)


def test_h_does_not_change_the_result_and_nothing_changes_twice():
    b = Batch(600, 1024, 300, 32, [0, 250], [0, 1], [32, 16], [1.0, 1.0])
    y, grads = b.forward(), b.backward()
    assert torch.equal(oq.lora_add(b.plan, b.x, b.A, b.B, b.base), y)
    for _ in range(3):
        assert torch.equal(b.forward(), y)
        assert all(torch.equal(p, q) for p, q in zip(b.backward(), grads))


def test_rows_that_are_not_finite_stay_alone():
    b = Batch(100, 128, 96, 8, [0, 40], [0, 1], [8, 5], [1.0, 1.0], F32)
    want, wdx = b.forward(), b.backward()[0]
    clean = torch.ones(100, dtype=torch.bool, device=DEV)
    clean[3] = clean[41] = clean[99] = False
    b.x[3, 7], b.x[99, 0] = float("nan"), float("inf")
    b.base[41, 5] = float("nan")
    got = b.forward()
    assert torch.equal(got[clean], want[clean])
    assert torch.isnan(got[3]).all() and not torch.isfinite(got[99]).any()
    assert torch.isnan(got[41, 5]) and torch.equal(got[41, 6:], want[41, 6:])
    b.x = torch.nan_to_num(b.x)
    b.forward()
    b.dy[3, 2], b.dy[41, 2], b.dy[99, 1] = float("nan"), float("inf"), float("nan")
    dx, dA, dB = b.backward()
    assert torch.equal(dx[clean][:, :], wdx[clean]) or torch.isfinite(dx[clean]).all()
    assert not torch.isfinite(dx[3]).any() and not torch.isfinite(dx[99]).any()


def test_one_adapter_does_not_touch_another():
    # rows of adapter 1 are not numbers; adapter 0's outputs and gradients are what they were
    b = Batch(200, 136, 72, 16, [0, 64, 100, 164], [0, 1, 0, 1], [16, 16], [1.0, 1.0])
    y, (dx, dA, dB) = b.forward(), b.backward()
    mine = torch.zeros(200, dtype=torch.bool, device=DEV)
    mine[:64] = mine[100:164] = True
    b.x[~mine], b.dy[~mine], b.base[~mine] = float("nan"), float("inf"), float("nan")
    b.A[1], b.B[1] = float("nan"), float("inf")
    y2, (dx2, dA2, dB2) = b.forward(), b.backward()
    assert torch.equal(y2[mine], y[mine]) and torch.equal(dx2[mine], dx[mine])
    assert torch.equal(dA2[0], dA[0]) and torch.equal(dB2[0], dB[0])


def test_empty_batch():
    plan = oq.lora_plan(0, [0, 0], [0, -1], [8], [1.0])
    A, B = _randn((1, 8, 16), 1), _randn((1, 5, 8), 2)
    e = lambda n, t=BF16: torch.empty((0, n), dtype=t, device=DEV)  # noqa: E731
    assert oq.lora_add(plan, e(16), A, B, e(5)).shape == (0, 5)
    dx, dA, dB = oq.lora_add_backward(plan, e(5), e(16), A, B, e(8, F32))
    assert dx.shape == (0, 16) and (dA == 0).all() and (dB == 0).all()


def test_many_adapters():
    n = 300
    r = np.random.default_rng(5)
    b = Batch(700, 64, 40, 8, sorted(r.integers(0, 700, 400).tolist()), r.integers(-1, n, 400).tolist(), r.integers(0, 9, n).tolist(),
              r.uniform(-1, 1, n).astype(np.float32).tolist())
    b.check_forward(b.forward())
    b.check_backward(*b.backward())


@pytest.mark.parametrize("M,stride", [(70, 2 ** 26 + 8), (3, 2 ** 31 + 1)])
def test_offsets_beyond_32_bits(M, stride):
    b = Batch(M, 136, 72, 16, [0, 1], [1, 0], [16, 9], [1.0, 0.5])
    want = (b.forward(),) + tuple(b.backward())

    def apart(t):
        wide = torch.empty(stride * (M - 1) + t.shape[1], dtype=t.dtype, device=DEV).as_strided(t.shape, (stride, 1))
        return wide.copy_(t)

    b.x, b.dy, b.base = apart(b.x), apart(b.dy), apart(b.base)
    assert torch.equal(b.forward(out=b.base), want[0]) and torch.equal(b.base, want[0])
    base = apart(torch.zeros_like(want[1]))
    dx, dA, dB = b.backward(base=base, out=base)
    assert torch.equal(base, want[1]) and torch.equal(dx, want[1]) and torch.equal(dA, want[2]) and torch.equal(dB, want[3])


def test_streams_and_graph_replays():
    b = Batch(300, 520, 264, 16, [0, 100], [0, 1], [16, 9], [1.0, 0.5])

    def call():
        return (b.forward(),) + tuple(b.backward())

    want = call()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = call()
    stream.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in (30, 40, 50):
        b.x.copy_(_randn(b.x.shape, seed))
        b.dy.copy_(_randn(b.dy.shape, seed + 1))
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want))


def test_beside_the_quantized_projection():
    # as it is used: the quantized layer's output, then the adapters on the layer's own input
    M, K, N = 96, 512, 384
    X, W = _randn((M, K), 60), _randn((N, K), 61, K ** -0.5)
    rot, cb = oq.rpbh_plan(K, 128, 0), oq.lloydmax_codebook(4, K)
    wc, wn = oq.quantize_weights_offline(rot, cb, W)
    xc, xn = oq.rpbh_quantize_act(rot, cb, X)
    b = Batch(M, K, N, 16, [0, 30], [0, 1], [16, 8], [1.0, 1.0], F32)
    b.x, b.base = X, oq.orbit_qlinear(cb, xc, xn, cb, wc, wn)
    b.check_forward(b.forward())


def test_refusals():
    b = Batch(20, 64, 48, 8, [0, 10], [0, 1], [8, 4], [1.0, 1.0])

    def refused(call, *words):
        with pytest.raises((ValueError, oq.OrbitError)) as e:
            call()
        assert all(word in str(e.value) for word in words), str(e.value)

    add = lambda plan=b.plan, x=b.x, A=b.A, B=b.B, base=b.base, **kw: oq.lora_add(plan, x, A, B, base, **kw)  # noqa: E731
    back = lambda dy=b.dy, x=b.x, h=b.h, **kw: oq.lora_add_backward(b.plan, dy, x, b.A, b.B, h, **kw)  # noqa: E731
    refused(lambda: add(plan=None), "plan")
    refused(lambda: add(x=b.x[:19]), "19 rows")
    refused(lambda: add(x=b.x.float()), "bf16")
    refused(lambda: add(x=b.x.cpu()), "GPU")
    refused(lambda: add(x=b.x[:, ::2]), "contiguous")
    refused(lambda: add(A=b.A[:1]), "A")
    refused(lambda: add(A=b.A[:, :, :32]), "A")
    refused(lambda: add(A=b.A.float()), "A")
    refused(lambda: add(B=b.B[:, :, :4]), "B")
    refused(lambda: add(B=b.B[0]), "3-D")
    refused(lambda: add(base=b.base[:, :40]), "base")
    refused(lambda: add(base=b.base.half()), "base")
    refused(lambda: add(base=b.base.cpu()), "base")
    refused(lambda: add(base=None), "base")
    refused(lambda: add(out=torch.empty_like(b.base, dtype=F32)), "out")
    refused(lambda: add(out=b.base[:1].expand(20, 48)), "overlap")
    refused(lambda: add(h=torch.empty((20, 4), dtype=F32, device=DEV)), "h")
    refused(lambda: add(h=b.h.to(BF16)), "h")
    refused(lambda: back(dy=b.dy.float()), "dY")
    refused(lambda: back(dy=b.dy[:, :47]), "dY")
    refused(lambda: back(h=b.h[:10]), "h")
    refused(lambda: back(base=b.dy), "base")
    refused(lambda: add(A=_randn((2, 12, 64), 1), B=_randn((2, 48, 12), 1)), "R=12")
    refused(lambda: add(A=_randn((2, 136, 64), 1), B=_randn((2, 48, 136), 1)), "R=136")
    refused(lambda: add(x=_randn((20, 60), 1), A=_randn((2, 8, 60), 1)), "K=60")
    sixteen = oq.lora_plan(20, [0], [0], [16, 2], [1.0, 1.0])
    refused(lambda: add(plan=sixteen), "rank 16")


# --- the kernels' other ways ----------------------------------------------------------------------
@pytest.mark.parametrize("R,ranks", [(8, [8, 5]), (16, [16, 3]), (24, [17, 24]), (32, [32, 31]), (48, [33, 48]), (64, [64, 1]), (80, [65, 80]),
                                     (128, [128, 100])])
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_rows_of_many_requests(R, ranks, rows, dtype):
    # both products in one kernel: requests of up to 4 rows, some without an adapter, an output of odd stride
    for K, N in ((8, 3), (520, 1111), (3072, 700)):
        M = 7 * rows
        b = Batch(M, K, N, R, [rows * i for i in range(7)], [0, 1, -1, 1, 0, 0, 1], ranks, [0.5, -2.0], dtype)
        whole = torch.full((M, N + 3), 7.0, dtype=dtype, device=DEV)
        y = b.forward(out=whole[:, 1:1 + N])
        b.check_forward(y)
        b.check_h(b.h)
        assert (whole[:, :1] == 7).all() and (whole[:, 1 + N:] == 7).all()
        in_place = b.base.clone()
        assert torch.equal(oq.lora_add(b.plan, b.x, b.A, b.B, in_place, out=in_place), y)
        b.check_backward(*b.backward())
        if N == 700:
            names = [r.kernel for r in launches(lambda: b.forward(out=y))]
            assert len(names) == 1 and "lora_rows_kernel" in names[0]


def test_few_rows_that_are_not_finite():
    b = Batch(6, 520, 100, 16, [0, 1, 2, 4], [0, 1, 0, 1], [16, 9], [1.0, 1.0], F32)
    want = b.forward()
    b.x[1, 519] = float("inf")
    b.x[3, 0] = float("nan")
    b.base[4, 7] = float("nan")
    got = b.forward()
    assert torch.equal(got[[0, 2, 5]], want[[0, 2, 5]])
    assert not torch.isfinite(got[1]).any() and torch.isnan(got[3]).all()
    assert torch.isnan(got[4, 7]) and torch.equal(got[4, 8:], want[4, 8:])


@pytest.mark.parametrize("R,rank", [(8, 7), (32, 32), (64, 50), (128, 128), (72, 72)])
@pytest.mark.parametrize("N", [384, 385, 511])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_whole_tiles(R, rank, N, dtype):
    # tiles of 64 rows, widths in whole strips and not, a contraction of whole chunks and not
    for K in (1024, 1096):
        b = Batch(256, K, N, R, [0, 128], [0, 1], [rank, rank], [1.0, 0.5], dtype)
        b.check_forward(b.forward())
        b.check_backward(*b.backward())


def _on_device(b):
    """The oracle's formulas in fp64 on the device, for batches that numpy would take long over."""
    x, dy, A, B = (torch.nan_to_num(t).double() for t in (b.x, b.dy, b.A, b.B))
    refs = [b.base.double(), torch.zeros_like(x), torch.zeros_like(A), torch.zeros_like(B)]
    sizes = [torch.zeros_like(r) for r in refs]
    starts = b.lists["starts"]
    for first, end, a in zip(starts, starts[1:] + [b.M], b.lists["adapters"]):
        s = b.lists["scales"][a]
        for out, f in ((refs, lambda t: t), (sizes, torch.abs)):
            xs, ds, Aa, Ba, sc = f(x[first:end]), f(dy[first:end]), f(A[a]), f(B[a]), abs(s) if f is torch.abs else s
            h, g = xs @ Aa.t(), ds @ Ba
            out[0][first:end] += sc * h @ Ba.t()
            out[1][first:end] += sc * g @ Aa
            out[2][a] += sc * g.t() @ xs
            out[3][a] += sc * ds.t() @ h
    return refs, sizes


@pytest.mark.parametrize("M,K,N,R,starts,adapters,ways", [
    (1000, 256, 392, 16, [0, 500], [0, 1], "lora_grad_kernel<1,false>"),              # more than 4 tiles to an adapter
    (16384 + 40, 2048, 2056, 8, [0], [0], "lora_grad_kernel<1,true>"),                # waves that share columns, partial sums
    (16384 + 33, 2048, 2049, 64, [0, 8000], [1, 0], "lora_grad_kernel<4,true>"),
    (300, 520, 770, 128, [0, 150], [0, 1], "lora_grad_kernel<4,true>"),               # at most 4 tiles: no partial sums
    (1500, 520, 770, 96, [0], [0], "lora_grad_kernel<4,false>"),
])
def test_ways_of_the_gradients(M, K, N, R, starts, adapters, ways):
    b = Batch(M, K, N, R, starts, adapters, [R, R - 1], [0.5, -1.0])
    y = b.forward()
    dx, dA, dB = b.backward()
    refs, sizes = _on_device(b)
    grow = (10 * max(K, N) ** 0.5 + 120) * U
    for name, got, ref, size, bar in (("y", y, refs[0], sizes[0], HALF_ULP[BF16]), ("dx", dx, refs[1], sizes[1], HALF_ULP[BF16]),
                                      ("dA", dA, refs[2], sizes[2], U), ("dB", dB, refs[3], sizes[3], U)):
        more = grow + 10 * M ** 0.5 * U if name in ("dA", "dB") else grow
        over = ((got.double() - ref).abs() - (bar * ref.abs() + (2.0 ** -16 + more) * size + 2 * U * ref.abs())).max()
        assert float(over) <= 0.0, f"{name}: {float(over)} beyond its bar"
    assert any(r.kernel == ways for r in launches(lambda: b.backward(out=dx)))


# --- all bits of the narrow sums ------------------------------------------------------------------
# 1 + 2^-10 + 2^-20 takes three bf16 values: what a result keeps of it once 1 + 2^-10 is taken off again is 2^-20, exactly,
# in sums of any order (every partial sum has at most 22 bits), and nothing at all where only two values were multiplied
WHOLE = 1 + 2.0 ** -10 + 2.0 ** -20
ALL = slice(None)


def _set(shape, *values):
    t = torch.zeros(shape, dtype=BF16, device=DEV)
    for at, v in values:
        t[at] = v
    return t


@pytest.mark.parametrize("M", [3, 70, 200])
@pytest.mark.parametrize("R,first,second", [(8, 0, 7), (32, 3, 20), (48, 1, 40), (64, 40, 50), (128, 2, 127), (128, 70, 71)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_have_all_bits_of_h(M, R, first, second, dtype):
    K, N = 264, 300
    plan = oq.lora_plan(M, [0], [0], [R], [0.5])
    x = _set((M, K), ((ALL, 0), 1.0), ((ALL, 130), 2.0 ** -10), ((ALL, 263), 2.0 ** -20))
    A = _set((1, R, K), ((0, first), 1.0), ((0, second, 0), 1.0), ((0, second, 130), 1.0))
    B = _set((1, N, R), ((0, ALL, first), 1.0), ((0, ALL, second), -1.0))
    h = torch.empty((M, R), dtype=F32, device=DEV)
    y = oq.lora_add(plan, x, A, B, torch.zeros((M, N), dtype=dtype, device=DEV), h=h)
    assert (h[:, first] == WHOLE).all() and (h[:, second] == 1 + 2.0 ** -10).all()
    assert (y == 0.5 * 2.0 ** -20).all()


@pytest.mark.parametrize("M", [3, 70, 2000])
@pytest.mark.parametrize("R,first,second", [(8, 0, 7), (32, 3, 20), (48, 1, 40), (64, 40, 50), (128, 2, 127), (128, 70, 71)])
def test_gradients_have_all_bits_of_h_and_g(M, R, first, second):
    K, N = 264, 300
    plan = oq.lora_plan(M, [0], [0], [R], [0.5])
    dy = _set((M, N), ((ALL, 0), 1.0), ((ALL, 130), 2.0 ** -10), ((ALL, 299), 2.0 ** -20))
    B = _set((1, N, R), ((0, ALL, first), 1.0), ((0, 0, second), 1.0), ((0, 130, second), 1.0))
    A = _set((1, R, K), ((0, first), 1.0), ((0, second), -1.0))
    one, x = torch.zeros((M, R), dtype=F32, device=DEV), torch.zeros((M, K), dtype=BF16, device=DEV)
    dx, _, _ = oq.lora_add_backward(plan, dy, x, A, B, one)
    assert (dx == 0.5 * 2.0 ** -20).all()
    # two rows whose contributions differ in the last bits alone
    last = M - 1
    dy[1:last], dy[last], x[0], x[last] = 0.0, -dy[0], 1.0, 1.0
    dy[last, 299] = 0.0
    _, dA, _ = oq.lora_add_backward(plan, dy, x, A, B, one)
    assert (dA[0, first] == 0.5 * 2.0 ** -20).all()
    one[0, first], one[last, first] = WHOLE, 1 + 2.0 ** -10
    dy.zero_()
    dy[0], dy[last] = 1.0, -1.0
    _, _, dB = oq.lora_add_backward(plan, dy, x, A, B, one)
    assert (dB[0, :, first] == 0.5 * 2.0 ** -20).all()


@pytest.mark.parametrize("M,K,N,R,ways", [(100, 128, 96, 8, "lora_grad_kernel<1,true>"), (1000, 256, 392, 16, "lora_grad_kernel<1,false>"),
                                          (16384 + 40, 2048, 2056, 8, "lora_grad_kernel<1,true>"), (300, 520, 770, 128, "lora_grad_kernel<4,true>"),
                                          (1500, 520, 770, 96, "lora_grad_kernel<4,false>")])
def test_gradients_beyond_the_ranks_are_zeros_whatever_x_and_dy_hold(M, K, N, R, ways):
    ranks, half = [R - 3, R], M // 2
    b = Batch(M, K, N, R, [0, half], [0, 1], ranks, [0.5, -1.0])
    b.forward()
    want = b.backward()
    b.x[3, 7], b.x[half - 1, K - 1] = float("nan"), float("inf")
    b.dy[5, 2], b.dy[half - 2, N - 1] = float("-inf"), float("nan")
    dx, dA, dB = b.backward()
    hit = torch.zeros(M, dtype=torch.bool, device=DEV)
    hit[5] = hit[half - 2] = True
    # the rows that hold them, their columns of the adapter's own gradients (dA's all: g of those rows is not finite), and no more
    assert torch.equal(dx[~hit], want[0][~hit]) and not torch.isfinite(dx[hit]).any()
    assert not torch.isfinite(dA[0, :R - 3]).any() and (dA[0, R - 3:] == 0).all() and torch.equal(dA[1], want[1][1])
    poisoned = torch.zeros(N, dtype=torch.bool, device=DEV)
    poisoned[2] = poisoned[N - 1] = True
    assert not torch.isfinite(dB[0, poisoned, :R - 3]).any() and torch.equal(dB[0, ~poisoned], want[2][0, ~poisoned])
    assert (dB[0, :, R - 3:] == 0).all() and torch.equal(dB[1], want[2][1])
    assert any(r.kernel == ways for r in launches(lambda: b.backward(out=dx)))


def test_gradients_of_rows_that_are_not_finite_stay_with_them():
    b = Batch(100, 128, 96, 8, [0, 40], [0, 1], [8, 5], [1.0, 1.0], F32)
    b.forward()
    want = b.backward()
    b.dy[3, 2], b.dy[41, 2], b.dy[99, 1] = float("nan"), float("inf"), float("nan")
    dx, dA, dB = b.backward()
    clean = torch.ones(100, dtype=torch.bool, device=DEV)
    clean[3] = clean[41] = clean[99] = False
    assert torch.equal(dx[clean], want[0][clean]) and not torch.isfinite(dx[~clean]).any()
    assert not torch.isfinite(dA[0]).any() and not torch.isfinite(dA[1, :5]).any() and (dA[1, 5:] == 0).all()
    assert not torch.isfinite(dB[0, 2]).any() and not torch.isfinite(dB[1, 1:3, :5]).any() and (dB[1, :, 5:] == 0).all()
    assert torch.equal(dB[0, 3:], want[2][0, 3:]) and torch.equal(dB[1, 3:], want[2][1, 3:])


@pytest.mark.parametrize("M", [3, 70, 2000])
@pytest.mark.parametrize("R", [8, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sums_above_the_largest_bf16_value(M, R, dtype):
    # h and g of (2 - 2^-7) 2^127 + 2^119 + 2^118, which fp32 holds and whose nearest bf16 value is an infinity
    K, N, large = 264, 300, (2 - 2.0 ** -7) * 2.0 ** 127 + 2.0 ** 119 + 2.0 ** 118
    parts = ((ALL, 0), (2 - 2.0 ** -7) * 2.0 ** 127), ((ALL, 130), 2.0 ** 119), ((ALL, 263), 2.0 ** 118)
    plan = oq.lora_plan(M, [0], [0], [R], [1.0])
    x, dy = _set((M, K), *parts), _set((M, N), *parts)
    wide_a, wide_b = _set((1, R, K), ((0, 1), 1.0)), _set((1, N, R), ((0, ALL, 1), 1.0))
    thin_a, thin_b = _set((1, R, K), ((0, 1), 2.0 ** -100)), _set((1, N, R), ((0, ALL, 1), 2.0 ** -100))
    h = torch.empty((M, R), dtype=F32, device=DEV)
    y = oq.lora_add(plan, x, wide_a, thin_b, torch.zeros((M, N), dtype=dtype, device=DEV), h=h)
    assert (h[:, 1] == large).all()
    want = torch.tensor(large * 2.0 ** -100, dtype=F32, device=DEV)
    assert (y == want.to(dtype)).all()
    if dtype == F32:
        return
    dx, _, _ = oq.lora_add_backward(plan, dy, x, thin_a, wide_b, h)
    assert (dx == want.to(BF16)).all()
    # one row's g and h alone
    x.zero_()
    dy[1:] = 0.0
    x[0] = 2.0 ** -100
    _, dA, _ = oq.lora_add_backward(plan, dy, x, thin_a, wide_b, h)
    assert (dA[0, 1] == want).all()
    dy[0] = 2.0 ** -100
    _, _, dB = oq.lora_add_backward(plan, dy, x, thin_a, wide_b, h)
    assert (dB[0, :, 1] == want).all()


def test_many_short_requests_on_wide_rows():
    # more tiles times columns than a grid of 512 columns to a workgroup holds; every request's row is one of B's columns
    M, K, N = 467_000, 8, 18432
    starts = list(range(M - 4))                                  # the last request has 5 rows
    adapters = [i % 2 for i in range(M - 4)]
    plan = oq.lora_plan(M, starts, adapters, [8, 8], [1.0, 1.0])
    m = torch.arange(M, device=DEV)
    x = torch.nn.functional.one_hot(m % 8, 8).to(BF16)
    A = torch.eye(8, dtype=BF16, device=DEV).expand(2, 8, 8).contiguous()
    n, r = torch.arange(N, device=DEV)[:, None], torch.arange(8, device=DEV)
    B = torch.stack([((n + 3 * r + 5 * a) % 101).to(BF16) for a in range(2)])
    y = torch.zeros((M, N), dtype=BF16, device=DEV)
    oq.lora_add(plan, x, A, B, y, out=y)
    rows = B.transpose(1, 2).reshape(16, N)
    which = torch.tensor(adapters + adapters[-1:] * 4, device=DEV) * 8 + m % 8
    for at in range(0, M, 8192):
        assert torch.equal(y[at:at + 8192], rows[which[at:at + 8192]])
