"""Plans of attention on the host, and what the entry points of attention and of the layer norms refuse before any launch (no
GPU work)."""

import contextlib
import ctypes
import types

import pytest
import torch

import paper_2607_02461_amd as oq
from paper_2607_02461_amd import norms


class Heads(ctypes.Structure):   # orbit_heads of the C header
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Rows(ctypes.Structure):    # orbit_rows
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("row", ctypes.c_int64), ("dtype", ctypes.c_int32)]


FAKE = [(1 << 30) + (i << 24) for i in range(9)]   # never dereferenced: every case fails its checks


@pytest.mark.parametrize("args,kw,word", [
    (([4], [4]), dict(heads=4, kv_heads=3), "heads"), (([4], [4]), dict(heads=0), "heads"), (([4], [4]), dict(heads=4, kv_heads=-2), "heads"),
    (([4], [4]), dict(heads=32768), "32767"), (([4, 4], [4]), dict(heads=1), "one length"), (([-1], [4]), dict(heads=1), "negative"),
    (([4], [-4]), dict(heads=1), "negative"), (([4], [4]), dict(heads=1, q_starts=[-1]), "negative"), (([4], [4]), dict(heads=1, k_starts=[1, 2]), "one length"),
    (([4.5], [4]), dict(heads=1), "whole numbers"), (([[4]], [[4]]), dict(heads=1), "whole numbers"), (([4],), dict(heads=1, k_starts=[0]), "without"),
    (([1 << 31], [4]), dict(heads=1), "2\\^31"), (([4], [1 << 31]), dict(heads=1), "2\\^31"), (([1 << 28], [4]), dict(heads=16, kv_heads=1), "2\\^31"),
    (([4], [4]), dict(heads=1, q_starts=[(1 << 31) - 2]), "2\\^31"), (([1 << 30], [4]), dict(heads=4), "tiles"), (([4], [1 << 30]), dict(heads=4), "tiles"),
    (([4, 4], [4, 4]), dict(heads=1, q_starts=[0, 3]), "query in common"), (([4, 4], [4, 4]), dict(heads=1 << 31), "32-bit"),
])
def test_plans_refuse(args, kw, word):
    with pytest.raises((ValueError, oq.OrbitError), match=word):
        oq.attention_plan(*args, **kw)


def test_plans_take():
    for args, kw in ((([], []), {}), (([0, 3], [5, 0]), {}), (([4, 4], [4, 4]), dict(q_starts=[4, 0], k_starts=[0, 0])),
                     (([1] * 1000, [9] * 1000), {}), (([1 << 24], [0]), dict(heads=1, q_starts=[(1 << 31) - 1 - (1 << 24)]))):
        plan = oq.attention_plan(*args, **{"heads": 4, "kv_heads": None if kw.get("heads") else 2, **kw})
        for backward in (0, 1):
            n = ctypes.c_size_t(7)
            assert oq.lib().attention_workspace_size(plan.handle, 128, backward, ctypes.byref(n)) == 0


def test_workspace_sizes():
    lib = oq.lib()

    def size(plan, D, backward):
        n = ctypes.c_size_t(7)
        return lib.attention_workspace_size(plan.handle, D, backward, ctypes.byref(n)), n.value

    many = oq.attention_plan([4096] * 4, heads=32)
    assert size(many, 128, 0) == (0, 0)                                        # enough tiles: no partial sums
    assert size(many, 128, 1) == (0, 2 * 4 * 32 * 4 * 4096)                    # lse and delta of each row
    few = oq.attention_plan([1], [4096], heads=8, kv_heads=1)
    assert size(few, 128, 0)[1] > 0 and size(few, 64, 0)[1] < size(few, 128, 0)[1]
    assert size(many, 132, 0) == (2, 0) and size(many, 0, 0) == (2, 0) and size(many, 136, 1) == (2, 0)
    n = ctypes.c_size_t(7)
    assert lib.attention_workspace_size(None, 128, 0, ctypes.byref(n)) == 1 and n.value == 0
    assert lib.attention_workspace_size(many.handle, 128, 0, None) == 1
    assert lib.attention_plan_upload(None) == 1
    lib.attention_plan_destroy(None)


def test_attention_validates_before_launch():
    lib = oq.lib()
    plan, split = oq.attention_plan([512] * 64, heads=4, kv_heads=2), oq.attention_plan([3], [4096], heads=4, kv_heads=2)

    def heads(i, data=None, token=None, head=64, n=None, dtype=1):
        n = (4 if i in (0, 3) else 2) if n is None else n
        return ctypes.byref(Heads(FAKE[i] if data is None else data, 0, n * head if token is None else token, head, n, dtype))

    def call(p=plan.handle, q=heads(0), k=heads(1), v=heads(2), o=heads(3), D=64, scale=0.125, lse=None, ws=None, n=0):
        return lib.attention(p, q, k, v, o, D, scale, lse, ws, n, None), lib.orbit_last_error().decode()

    cases = [
        (dict(p=None), 1, "plan"), (dict(D=60), 2, "head size"), (dict(D=136), 2, "head size"), (dict(scale=0.0), 1, "scale"), (dict(scale=-1.0), 1, "scale"),
        (dict(scale=float("nan")), 1, "scale"), (dict(scale=float("inf")), 1, "scale"), (dict(q=None), 1, "q is NULL"), (dict(o=None), 1, "out is NULL"),
        (dict(q=heads(0, n=2)), 1, "heads"), (dict(k=heads(1, n=4)), 1, "heads"), (dict(q=heads(0, dtype=0)), 1, "type"), (dict(v=heads(2, dtype=3)), 1, "type"),
        (dict(o=heads(3, dtype=5)), 1, "type"), (dict(q=heads(0, data=0)), 1, "null"), (dict(k=heads(1, data=FAKE[1] + 8)), 1, "16 bytes"),
        (dict(q=heads(0, token=252)), 1, "16 bytes"), (dict(k=heads(1, head=68)), 1, "16 bytes"), (dict(k=heads(1, token=-128)), 1, "range"),
        (dict(v=heads(2, token=(1 << 24) + 8)), 1, "range"), (dict(o=heads(3, token=128)), 1, "overlap"), (dict(o=heads(3, head=32)), 1, "overlap"),
        (dict(o=heads(0)), 1, "lies on"), (dict(o=heads(3, data=FAKE[2])), 1, "lies on"), (dict(lse=FAKE[4] + 2), 1, "lse"), (dict(p=split.handle), 1, "workspace"),
        (dict(p=split.handle, ws=FAKE[5], n=64), 1, "workspace"),
    ]
    for kw, status, word in cases:
        st, msg = call(**kw)
        assert st == status and word in msg, (kw, st, msg)
    assert lib.attention(oq.attention_plan([0], [3], heads=4).handle, None, None, None, None, 64, 1.0, None, None, 0, None) == 0   # no queries


def test_attention_backward_validates_before_launch():
    lib = oq.lib()
    plan = oq.attention_plan([40, 30], [50, 60], heads=4, kv_heads=2, causal=True)
    shared = oq.attention_plan([40, 30], [50, 60], heads=4, kv_heads=2, k_starts=[0, 10])

    def heads(i, data=None, n=None, dtype=1, head=64):
        n = (2 if i in (2, 3, 6, 7) else 4) if n is None else n
        return ctypes.byref(Heads(FAKE[i] if data is None else data, 0, 4 * 64, head, n, dtype))

    def call(p=plan.handle, g=heads(0), q=heads(1), k=heads(2), v=heads(3), o=heads(4), lse=1 << 20, dq=heads(5), dk=heads(6), dv=heads(7), D=64, scale=1.0,
             ws=FAKE[8], n=1 << 40):
        return lib.attention_backward(p, g, q, k, v, o, lse, dq, dk, dv, D, scale, ws, n, None), lib.orbit_last_error().decode()

    for kw, status, word in (
            (dict(p=None), 1, "plan"), (dict(p=shared.handle), 1, "key in common"), (dict(D=4), 2, "head size"), (dict(scale=0.0), 1, "scale"),
            (dict(g=None), 1, "dout"), (dict(g=heads(0, dtype=0)), 1, "type"), (dict(dk=heads(6, dtype=0)), 1, "type"), (dict(dv=heads(7, n=4)), 1, "heads"),
            (dict(dq=heads(1)), 1, "input"), (dict(dk=heads(6, data=FAKE[2])), 1, "input"), (dict(dv=heads(7, data=FAKE[6])), 1, "one place"),
            (dict(lse=None), 1, "lse"), (dict(lse=(1 << 20) + 1), 1, "lse"), (dict(ws=None), 1, "workspace"), (dict(n=1 << 10), 1, "workspace"),
            (dict(dq=heads(5, head=32)), 1, "overlap"), (dict(q=heads(1, head=1 << 30)), 2, "apart")):
        st, msg = call(**kw)
        assert st == status and word in msg, (kw, st, msg)


def test_layer_norm_validates_before_launch():
    lib = oq.lib()

    def rows(i, data=None, batch=640, row=64, dtype=1):
        return ctypes.byref(Rows(FAKE[i] if data is None else data, batch, row, dtype))

    def forward(x=rows(0), y=rows(1), B=2, L=10, N=64, w=FAKE[3], wb=0, b=FAKE[4], bb=0, wd=1, mod=0, eps=1e-6):
        return lib.layer_norm(x, y, B, L, N, w, wb, b, bb, wd, mod, eps, None), lib.orbit_last_error().decode()

    for kw, status, word in (
            (dict(x=None), 1, "x is NULL"), (dict(y=None), 1, "y is NULL"), (dict(x=rows(0, dtype=3)), 1, "type"), (dict(x=rows(0, data=0)), 1, "null"),
            (dict(y=rows(1, data=FAKE[1] + 1)), 1, "misaligned"), (dict(B=-1), 1, "negative"), (dict(N=0), 1, "N=0"), (dict(N=12289), 2, "12288"),
            (dict(B=1 << 16, L=1 << 16), 2, "2^31"), (dict(x=rows(0, row=-64)), 1, "range"), (dict(x=rows(0, batch=1 << 60)), 1, "range"),
            (dict(y=rows(1, row=63)), 1, "overlap"), (dict(y=rows(1, batch=639)), 1, "overlap"), (dict(y=rows(1, batch=64, row=64)), 1, "overlap"),
            (dict(y=rows(0, dtype=0)), 1, "row by row"), (dict(y=rows(0, row=72, batch=720)), 1, "row by row"), (dict(w=FAKE[3] + 1), 1, "misaligned"),
            (dict(wd=0, b=FAKE[4] + 2), 1, "misaligned"), (dict(wd=7), 1, "type"), (dict(bb=-1), 1, "range"), (dict(eps=-1.0), 1, "eps"),
            (dict(eps=float("nan")), 1, "eps"), (dict(eps=float("inf")), 1, "eps")):
        st, msg = forward(**kw)
        assert st == status and word in msg, (kw, st, msg)
    assert forward(B=0)[0] == 0 and forward(L=0, x=rows(0, data=0))[0] == 0

    def backward(g=rows(0), x=rows(1), dx=rows(2), B=2, L=10, N=64, w=FAKE[3], wb=0, wd=1, mod=0, eps=1e-6, dw=FAKE[4], db=FAKE[5], per=0, ws=FAKE[6], n=1 << 30):
        return lib.layer_norm_backward(g, x, dx, B, L, N, w, wb, wd, mod, eps, dw, db, per, ws, n, None), lib.orbit_last_error().decode()

    for kw, status, word in (
            (dict(g=None), 1, "dy is NULL"), (dict(dx=rows(2, dtype=0)), 1, "x's type"), (dict(dx=rows(0, batch=0, row=128)), 1, "overlap"),
            (dict(dx=rows(1, batch=1280, row=128)), 1, "row by row"), (dict(wb=64), 1, "gradients of their own"), (dict(dw=FAKE[4] + 2), 1, "misaligned"),
            (dict(eps=-1.0), 1, "eps"), (dict(N=20000), 2, "12288"), (dict(wd=9), 1, "type")):
        st, msg = backward(**kw)
        assert st == status and word in msg, (kw, st, msg)
    n = ctypes.c_size_t(7)
    assert lib.layer_norm_backward_workspace_size(1, 1, 0, 0, ctypes.byref(n)) == 1 and n.value == 0
    assert lib.layer_norm_backward_workspace_size(1, 1, 8, 0, None) == 1


@pytest.mark.parametrize("like", [
    torch.zeros(100).unfold(0, 64, 1), torch.zeros(200).unfold(0, 64, 1), torch.zeros(3, 100).unfold(1, 64, 1), torch.zeros(100).unfold(0, 64, 3),
    torch.zeros(1, 64).expand(5, 64), torch.zeros(2, 1, 64).expand(2, 7, 64), torch.zeros(7, 2, 64).transpose(0, 1), torch.zeros(2, 9, 1),
    torch.zeros(9, 2, 1).transpose(0, 1), torch.zeros(64, 1).t(), torch.zeros(2, 9, 70)[..., 3:67], torch.zeros(0, 9, 64)])
def test_new_outputs_of_layer_norms_are_rows(like):
    # whatever order the input's dimensions have in memory: contiguous rows that do not overlap
    assert like.stride(-1) == 1 or like.shape[-1] == 1
    out, _ = norms._output(None, like, "out", torch.bfloat16)
    assert out.shape == like.shape and out.dtype == torch.bfloat16 and out.stride(-1) == 1
    reach = 0
    for stride, size in sorted(zip(out.stride(), out.shape)):
        if size > 1:
            assert stride > reach
            reach += stride * (size - 1)


@pytest.mark.parametrize("known", [False, True])
def test_workspace_sizes_survive_another_threads_clearing(monkeypatch, known):
    # the list of known sizes is emptied when it is long; another thread may do so between any two steps of this one
    class Emptied(dict):
        def __contains__(self, key):
            found = super().__contains__(key)
            self.clear()
            return found

        def __setitem__(self, key, value):
            super().__setitem__(key, value)
            self.clear()

    def size(B, L, N, per_batch, out):
        out._obj.value = 48
        return 0

    cpu = torch.device("cpu")
    sizes = Emptied()
    if known:
        dict.__setitem__(sizes, (1, 2, 3, 0, cpu), 48)
    monkeypatch.setattr(norms, "_workspace_bytes", sizes)
    monkeypatch.setattr(norms, "lib", lambda: types.SimpleNamespace(layer_norm_backward_workspace_size=size))
    monkeypatch.setattr(torch.cuda, "device", lambda dev: contextlib.nullcontext())
    ws, n = norms._workspace(1, 2, 3, 0, cpu)
    assert n == 48 and ws.numel() == 48


@pytest.mark.parametrize("scale,backward", [(2.4e38, 0), (3.4e38, 0), (3.4e38, 1), (1e-38, 1), (1e-45, 1), (5e-31, 1)])
def test_scales_whose_scores_leave_fp32_are_refused(scale, backward):
    # forward, scores in units of log 2 are scale * 1.44; the backward pass measures rows' sums in units of scores, lse / scale
    plan = oq.attention_plan([40], [50], heads=4, kv_heads=2)

    def heads(i, n):
        return ctypes.byref(Heads(FAKE[i], 0, n * 64, 64, n, 1))

    q, k, v, out, dout, dq, dk, dv = (heads(i, n) for i, n in enumerate((4, 2, 2, 4, 4, 4, 2, 2)))
    if backward:
        st = oq.lib().attention_backward(plan.handle, dout, q, k, v, out, 1 << 20, dq, dk, dv, 64, scale, FAKE[8], 1 << 40, None)
    else:
        st = oq.lib().attention(plan.handle, q, k, v, out, 64, scale, None, None, 0, None)
    assert st == 2 and "scale" in oq.lib().orbit_last_error().decode()
