"""Plans of low-rank adapters on the host, and what the entry points refuse before any launch (no GPU work)."""

import ctypes

import pytest

import paper_2607_02461_amd as oq


def _plan(M=10, starts=(0, 4), adapters=(0, 1), ranks=(8, 8), scales=(1.0, 1.0)):
    return oq.lora_plan(M, starts, adapters, ranks, scales)


@pytest.mark.parametrize("kw,word", [
    (dict(M=-1), "negative"), (dict(M=1 << 31), "2\\^31"), (dict(starts=(4, 0)), "begins"), (dict(starts=(0, 11)), "begins"),
    (dict(starts=(-1, 4)), "begins"), (dict(starts=(0,)), "one length"), (dict(adapters=(0, 2)), "adapter 2"), (dict(adapters=(0, -2)), "adapter -2"),
    (dict(ranks=(8, -1)), "rank -1"), (dict(ranks=(8, 129)), "rank 129"), (dict(ranks=(8,)), "one length"), (dict(ranks=(), scales=()), "adapters"),
    (dict(scales=(1.0, float("nan"))), "finite"), (dict(scales=(1.0, 1e39)), "finite"), (dict(starts=(0.5, 4)), "starts"),
    (dict(starts=((0, 4),)), "starts"), (dict(starts=(0, 1 << 40)), "32-bit"), (dict(ranks=[1] * 70000, scales=[1.0] * 70000), "65535"),
    (dict(M=(1 << 31) - 1), "tiles"),
])
def test_plans_refuse(kw, word):
    with pytest.raises((ValueError, oq.OrbitError), match=word):
        _plan(**kw)


def test_plans_take():
    for kw in (dict(M=0, starts=(0, 0)), dict(starts=(), adapters=()), dict(starts=(10, 10)), dict(adapters=(-1, -1)), dict(ranks=(0, 128))):
        p = _plan(**kw)
        assert p.rows == kw.get("M", 10) and p.adapters == 2


def test_device_calls_validate_before_launch():
    lib, fake = oq.lib(), 1 << 20   # never dereferenced: every case fails validation first
    plan = _plan()

    def add(p=plan.handle, x=fake, ldx=64, a=fake, b=fake, K=64, N=32, R=8, base=fake, ldb=32, dtype=1, y=fake, ldy=32, h=None, ws=fake, n=1 << 30):
        return lib.lora_add(p, x, ldx, a, b, K, N, R, base, ldb, dtype, y, ldy, h, ws, n, None), lib.orbit_last_error().decode()

    for kw, status, word in (
            (dict(p=None), 1, "plan"), (dict(K=60), 1, "K=60"), (dict(K=0), 1, "K=0"), (dict(N=0), 1, "N=0"), (dict(R=4), 2, "R=4"),
            (dict(R=136), 2, "R=136"), (dict(K=1 << 22), 2, "above"), (dict(N=1 << 22), 2, "above"), (dict(dtype=3), 1, "type"),
            (dict(ldx=63), 1, "stride"), (dict(ldy=31), 1, "stride"), (dict(ldb=31), 1, "stride"), (dict(x=0), 1, "null"), (dict(b=0), 1, "null"),
            (dict(y=0), 1, "null"), (dict(a=fake + 8), 1, "misaligned"), (dict(x=fake + 1), 1, "misaligned"), (dict(h=fake + 4), 1, "misaligned")):
        st, msg = add(**kw)
        assert st == status and word in msg, (kw, st, msg)
    big = _plan(ranks=(8, 64))
    st, msg = add(p=big.handle)
    assert st == 1 and "rank 64" in msg
    st = lib.lora_add_backward(plan.handle, fake, 31, fake, 64, fake, fake, fake, 64, 32, 8, None, 0, fake, 64, fake, fake, fake, 1 << 30, None)
    assert st == 1 and "stride" in lib.orbit_last_error().decode()
    st = lib.lora_add_backward(plan.handle, fake, 32, fake, 64, fake, fake, fake, 64, 32, 8, None, 0, fake, 64, None, fake, fake, 1 << 30, None)
    assert st == 1 and "null" in lib.orbit_last_error().decode()
    n = ctypes.c_size_t(7)
    assert lib.lora_add_workspace_size(None, 64, 32, 8, 0, ctypes.byref(n)) == 1 and n.value == 0
    assert lib.lora_plan_upload(None) == 1
    lib.lora_plan_destroy(None)


def test_outputs_on_inputs_that_they_do_not_replace_are_refused():
    lib, at = oq.lib(), [1 << 20 + i for i in range(8)]   # never dereferenced: every case fails its checks
    plan = _plan()

    def refused(status, word):
        return status == 1 and word in lib.orbit_last_error().decode()

    def add(x, base, ldb, y, ldy):
        return lib.lora_add(plan.handle, x, 64, at[6], at[7], 64, 64, 8, base, ldb, 1, y, ldy, None, at[5], 1 << 30, None)

    assert refused(add(at[0], at[1], 64, at[1], 72), "another row stride")
    assert refused(add(at[0], at[1], 64, at[0], 64), "other than base")

    def back(dy, x, base, ldb, dx, lddx):
        return lib.lora_add_backward(plan.handle, dy, 64, x, 64, at[6], at[7], at[5], 64, 64, 8, base, ldb, dx, lddx, at[4], at[4], at[4], 1 << 30, None)

    assert refused(back(at[0], at[1], at[2], 64, at[2], 72), "another row stride")
    assert refused(back(at[0], at[1], None, 0, at[0], 64), "other than base")
    assert refused(back(at[0], at[1], at[2], 64, at[1], 64), "other than base")
