"""Registers and scratch of the kernels on whole caches, as the built library's metadata states them (no GPU needed)."""
import re

from tests.test_kernel_resources import kernels  # noqa: F401  (the fixture)


def test_nothing_in_scratch_and_room_for_the_waves_that_grids_are_shaped_for(kernels):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.search(r"span_(rows|f32|tiles|q4|merge)_kernel|append_kernel|read_rows_kernel", k)}
    assert len(found) > 20
    for name, (regs, scratch) in found.items():
        assert scratch == 0, name
        if q4 := re.search(r"span_q4_kernelINS_(4BF16|3F32)ELi(\d)E", name):
            waves = {"4": 4 if q4[1] == "4BF16" else 3}.get(q4[2], 2)
        elif "span_f32_kernelILi1E" in name:
            waves = 3
        elif "span_" in name and "merge" not in name:
            waves = 2
        else:
            continue
        assert regs <= 512 // waves // 8 * 8, name
