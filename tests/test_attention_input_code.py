"""What the compiler made of the kernels of the attention's input and of the adapters, read off the built library."""

import re

import pytest

from tests import code_objects


@pytest.fixture
def kernels(monkeypatch):
    # mangled names: instances differ in types, which the short names leave out
    monkeypatch.setattr(code_objects, "short_name", str)
    return code_objects.kernel_metadata()


# instances: layouts x non-temporal x types (and rows in flight); ranks x types x base; ranks x types x rows
@pytest.mark.parametrize("name,instances", [("axial_rope_kernel", 24), ("qk_norm_rope_backward_kernel", 32), ("norm_weight_grad_kernel", 1),
                                            ("lora_shrink_kernel", 4), ("lora_expand_kernel", 12), ("lora_rows_kernel", 20),
                                            ("lora_turn_kernel", 1), ("lora_grad_kernel", 6), ("lora_grad_sum_kernel", 1)])
def test_rows_and_sums_stay_in_registers(kernels, name, instances):
    mine = {n: k for n, k in kernels.items() if re.search(rf"\d{name}[EI]", n)}
    assert len(mine) == instances
    for n, k in mine.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, f"{n} spills"
