"""Workgroups of four waves that a CU's registers hold, of the kernels whose figures depend on it: 512 registers a lane of a SIMD, given out in eights.
No GPU needed."""
import os

import pytest

from paper_2605_22428_amd import build
from test_kernel_resources import _device_elf, _kernels

HELD = {"k_adapt_upILi1ELi1E": 5, "k_adapt_upILi1ELi2E": 4, "k_adapt_upILi2ELi1E": 4, "k_adapt_upILi2ELi2E": 3, "k_adapt_upILi4ELi1E": 3,
        "k_adapt_upILi4ELi2E": 2, "k_adapt_upILi8ELi1E": 1, "k_adapt_upILi8ELi2E": 1, "k_adapt_gradsILi1E": 3, "k_adapt_gradsILi2E": 1,
        "k_layer_upILb0ELb0E": 3, "k_layer_upILb0ELb1E": 2, "k_layer_upILb1ELb0E": 2, "k_layer_downILb0ELb0E": 3, "k_layer_downILb0ELb1E": 2,
        "k_layer_downILb1ELb0E": 2}


@pytest.fixture(scope="module")
def registers():
    path = build.LIB if os.path.exists(build.LIB) else build.build()
    return {k[".name"]: k[".vgpr_count"] for elf in _device_elf(path) for k in _kernels(elf)}


@pytest.mark.parametrize("kernel", sorted(HELD))
def test_workgroups_that_registers_hold(registers, kernel):
    found = [n for name, n in registers.items() if kernel in name]
    assert len(found) == 1
    assert 512 // (-(-found[0] // 8) * 8) >= HELD[kernel], found
