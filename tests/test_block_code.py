"""What the compiler made of the kernels of the layer norms and of attention, read off the built library."""

import re

import pytest

from tests import code_objects


@pytest.fixture
def kernels(monkeypatch):
    # mangled names: instances differ in types, which the short names leave out
    monkeypatch.setattr(code_objects, "short_name", str)
    return code_objects.kernel_metadata()


# instances: types x pieces x ways of a row's end; head sizes x workgroup sizes
@pytest.mark.parametrize("name,instances", [("layer_norm_kernel", 48), ("layer_norm_backward_kernel", 48), ("layer_norm_sum_kernel", 1),
                                            ("attention_kernel", 8), ("attention_few_kernel", 4), ("attention_join_kernel", 4),
                                            ("attention_row_grad_kernel", 4), ("attention_key_grad_kernel", 4), ("attention_grad_join_kernel", 4)])
def test_rows_and_sums_stay_in_registers(kernels, name, instances):
    mine = {n: k for n, k in kernels.items() if re.search(rf"\d{name}[EI]", n)}
    assert len(mine) == instances
    for n, k in mine.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, f"{n} spills"


# two workgroups of four waves to a compute unit, one of eight: two waves to a SIMD of 512 registers
@pytest.mark.parametrize("name", ["attention_kernel", "attention_row_grad_kernel", "attention_key_grad_kernel"])
def test_two_waves_fit_a_simd(kernels, name):
    for n, k in kernels.items():
        if re.search(rf"\d{name}I", n):
            assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 256, n
