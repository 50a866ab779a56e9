"""Plans of rotary positions on the host, and what the entry points refuse before any launch (no GPU work)."""

import ctypes

import numpy as np
import pytest

import paper_2607_02461_amd as oq


class Heads(ctypes.Structure):   # orbit_heads of the C header
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


@pytest.mark.parametrize("dims,lengths,word", [
    ((), (), "axes"), ((8,) * 9, (1,) * 9, "axes"), ((7, 9), (3, 3), "even"), ((0, 8), (3, 3), "even"), ((514,), (3,), "512"),
    ((8, 8), (3, 0), "positions"), ((8, 6), (3, 3), "multiple of 8"), ((512, 8), (3, 3), "multiple of 8"),
    ((512,), (1 << 20,), "exceed"), ((8, 8), (3,), "axes"), ((-8, 16), (3, 3), "32-bit"), ((8,), (1 << 31,), "32-bit"),
])
def test_plans_refuse(dims, lengths, word):
    with pytest.raises((ValueError, oq.OrbitError), match=word):
        oq.rope_plan(dims, lengths)


@pytest.mark.parametrize("theta", [0.0, -1.0, float("inf"), float("nan")])
def test_plans_refuse_theta(theta):
    with pytest.raises(oq.OrbitError, match="theta"):
        oq.rope_plan((8,), (4,), theta=theta)


def test_plans_refuse_angles():
    with pytest.raises(ValueError, match="angles"):
        oq.rope_plan_from_angles([])
    with pytest.raises(ValueError, match="angles"):
        oq.rope_plan_from_angles([np.zeros(8)])
    bad = np.zeros((3, 4))
    bad[2, 1] = np.inf
    with pytest.raises(oq.OrbitError, match="axis 0, position 2, pair 1"):
        oq.rope_plan_from_angles([bad])


def test_device_calls_validate_before_launch():
    lib, fake = oq.lib(), 1 << 20   # never dereferenced: every case fails validation first
    plan = oq.rope_plan((16, 16), (4, 4))

    def heads(data=fake, strides=(0, 64, 32), n=2, dtype=1):
        return ctypes.byref(Heads(data, *strides, n, dtype))

    def rope(plan=plan.handle, x=heads(), y=heads(), B=1, L=3, D=32, pos=fake, inverse=0):
        st = lib.axial_rope(plan, x, y, B, L, D, pos, 0, inverse, None)
        return st, lib.orbit_last_error().decode()

    for kw, status, word in (
            (dict(plan=None), 1, "plan"), (dict(x=None), 1, "x is NULL"), (dict(y=None), 1, "y is NULL"), (dict(x=heads(dtype=7)), 1, "type"),
            (dict(x=heads(n=0)), 1, "heads"), (dict(y=heads(n=3)), 1, "heads"), (dict(y=heads(dtype=0)), 1, "type"),
            (dict(x=heads(data=0)), 1, "null"), (dict(y=heads(data=fake + 8)), 1, "16 bytes"), (dict(x=heads(strides=(0, 60, 32))), 1, "16 bytes"),
            (dict(x=heads(strides=(0, -64, 32))), 1, "stride"), (dict(x=heads(strides=(0, 1 << 50, 32))), 1, "stride"),
            (dict(B=-1), 1, "negative"), (dict(D=36), 2, "head size"), (dict(D=1024), 2, "head size"), (dict(D=24), 1, "rotates 32"),
            (dict(pos=0), 1, "positions"), (dict(inverse=2), 1, "inverse"), (dict(L=1 << 30), 2, "head rows")):
        st, msg = rope(**kw)
        assert st == status and word in msg, (kw, st, msg)
    none = ctypes.c_void_p(0)
    st = lib.qk_norm_rope(plan.handle, heads(), heads(), heads(), none, 1, 3, 32, fake, 0, None, None, 0, 1e-6, None)
    assert st == 1 and "k_out" in lib.orbit_last_error().decode()
    st = lib.qk_norm_rope_backward(plan.handle, heads(), none, heads(), none, heads(), none, 1, 3, 32, fake, 0, None, None, 0, 1e-6, fake,
                                   None, None, 0, None)
    assert st == 1 and "without the weight" in lib.orbit_last_error().decode()
    assert lib.rope_plan_upload(None) == 1
    lib.rope_plan_destroy(None)


def test_outputs_on_inputs_that_they_do_not_replace_are_refused():
    lib, here, there = oq.lib(), 1 << 20, 1 << 24   # never dereferenced: without a device no call gets further than its checks
    plan = oq.rope_plan((16, 16), (4, 4))

    def heads(data, strides=(0, 64, 32), n=2, dtype=1):
        return ctypes.byref(Heads(data, *strides, n, dtype))

    def refused(status):
        return status == 1 and "lies on an input" in lib.orbit_last_error().decode()

    other = (0, 128, 32)
    rope = lambda x, y, L=3: lib.axial_rope(plan.handle, x, y, 1, L, 32, here, 0, 0, None)  # noqa: E731
    assert refused(rope(heads(here), heads(here, other)))
    none = ctypes.c_void_p(0)
    norm = lambda q, k, qo, ko: lib.qk_norm_rope(plan.handle, q, k, qo, ko, 1, 3, 32, here, 0, None, None, 0, 1e-6, None)  # noqa: E731
    assert refused(norm(heads(here, dtype=0), none, heads(here), none))                         # another type
    assert refused(norm(heads(here), heads(there), heads(there), heads(here)))                  # q and k change places
    assert refused(norm(heads(here), heads(here), heads(here), heads(there)))                   # q replaced, read as k
    assert refused(norm(heads(here), heads(here), heads(there), heads(there)))                  # one output for both
    back = lambda dq, q, qg, dk=none, k=none, kg=none: lib.qk_norm_rope_backward(  # noqa: E731
        plan.handle, dq, dk, q, k, qg, kg, 1, 3, 32, here, 0, None, None, 0, 1e-6, None, None, None, 0, None)
    assert refused(back(heads(here, dtype=0), heads(there), heads(here)))
    assert refused(back(heads(here), heads(there), heads(here, other)))
    assert refused(back(heads(here), heads(there), heads(2 * there), heads(3 * there), heads(4 * there), heads(here)))


@pytest.mark.parametrize("n,strides,B,status,word", [((1 << 31) - 1, (0, 1 << 34, 8), 1, 2, "heads"), ((1 << 30) + 1, (0, 1 << 34, 8), 1, 2, "heads"),
                                                     (2, (1 << 40, 64, 32), 1 << 20, 1, "stride"), (1 << 20, (0, 64, 1 << 40), 1, 1, "stride")])
def test_offsets_that_pass_their_numbers_are_refused(n, strides, B, status, word):
    # a token's last head and the rows behind it have 32-bit indices, an element's offset has 64 bits
    lib, plan = oq.lib(), oq.rope_plan((8,), (4,))
    x = ctypes.byref(Heads(1 << 20, *strides, n, 1))
    assert lib.axial_rope(plan.handle, x, x, B, 1, 8, 1 << 20, 0, 0, None) == status and word in lib.orbit_last_error().decode()
