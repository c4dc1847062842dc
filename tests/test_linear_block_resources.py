"""Registers and LDS of the linear-attention block's kernels: the workgroups a
CU (four SIMDs of 512 registers a lane, 160 KB of LDS) is meant to hold."""
import pytest

from test_kernel_resources import kernels  # noqa: F401  (fixture)

# Waves of a workgroup and workgroups per CU that a kernel's split was chosen for.
RESIDENT = {
    "la_chunk_kernelIDF16bLi128EE": (8, 2), "la_chunk_kernelIDF16bLi64EE": (4, 3),
    "la_chunk_kernelIfLi128EE": (8, 1), "la_chunk_kernelIfLi64EE": (4, 2),
    "la_state_kernelIDF16bLi128EE": (8, 2), "la_state_kernelIDF16bLi64EE": (4, 4),
    "la_state_kernelIfLi128EE": (8, 1), "la_state_kernelIfLi64EE": (4, 2),
    "la_step_kernelIDF16bLi128EE": (4, 8), "la_step_kernelIfLi128EE": (4, 8),
    "residual_norm_kernelILi2ELi3EDF16bDF16bEE": (2, 6),
    "residual_norm_kernelILi8ELi4EffEE": (8, 1),
    "linear_w4_kernelIDF16bDF16bLi128ELi1ELi1EE": (16, 2),
    "linear_w4_kernelIffLi32ELi1ELi1EE": (16, 1),
    "linear_w4_kernelIDF16bDF16bLi128ELi4ELi2EE": (8, 1),
    "linear_w4_kernelIffLi32ELi4ELi2EE": (8, 1),
}


@pytest.mark.parametrize("name", RESIDENT)
def test_workgroups_per_cu(kernels, name):  # noqa: F811
    waves, groups = RESIDENT[name]
    found = [k for ks in kernels.values() for k in ks if name in k["name"]]
    assert found, name
    for k in found:
        regs = int(k["vgpr_count"])  # accumulators included
        per_simd = -(-waves * groups // 4)
        assert -(-regs // 8) * 8 * per_simd <= 512, (k["name"], regs)
        assert int(k["group_segment_fixed_size"]) * groups <= 160 * 1024, k["name"]
        assert int(k["private_segment_fixed_size"]) == 0 and int(k["vgpr_spill_count"]) == 0
