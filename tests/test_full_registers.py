"""Registers of the kernels of full attention and rotary positions, from the built library (CPU only)."""
import re

import pytest

from test_kernel_registers import kernel_figures


@pytest.fixture(scope="module")
def figures(tmp_path_factory):
    found = kernel_figures(tmp_path_factory.mktemp("kernels"))
    return {s: f for s, f in found.items() if re.search(r"full_(fwd|dq|dkv|join|sum)_kernel|rotary_kernel", s)}


def test_no_spills(figures):
    """Of 360 kernels two (dK/dV at d = 64, d_V = 128, two groups) spill one register, outside their loops."""
    assert len(figures) == 360
    spilled = {s: (f[".vgpr_spill_count"], f[".sgpr_spill_count"], f[".private_segment_fixed_size"]) for s, f in figures.items()}
    assert {s: x for s, x in spilled.items() if x[0] > 1 or x[1] or x[2] > 8} == {}
    assert sum(x[0] > 0 for x in spilled.values()) <= 2


def test_two_waves_a_simd(figures):
    """Tiles of 128 rows are built for eight waves a CU at least: 256 registers, and LDS for two workgroups of four waves or one of
    eight; runs' plans count on it."""
    for s, f in figures.items():
        m = re.search(r"full_(?:fwd|dq|dkv)_kernelINS_4\w{4}ELi\d+ELi\d+ELi128ELi(\d)E", s)
        if m:
            assert f[".vgpr_count"] <= 256, s
            assert f[".group_segment_fixed_size"] * (2 if m.group(1) == "1" else 1) <= 160 * 1024, s
