"""Registers and LDS of the 8-bit block's kernels: the workgroups a CU (four SIMDs of 512 registers
a lane, 160 KB of LDS) is meant to hold."""
import pytest

from test_kernel_resources import kernels  # noqa: F401  (fixture)

# Waves of a workgroup and workgroups per CU that a kernel's split was chosen for.
RESIDENT = {"4TileILi4ELi2ELi4ELi8ELi1EE": (8, 1), "4TileILi2ELi2ELi4ELi4ELi2EE": (4, 2), "4TileILi4ELi1ELi1ELi4ELi4EE": (4, 4),
            "ELi8ELi2ELi1EEEv": (8, 2), "ELi8ELi2ELi2EEEv": (8, 2), "ELi8ELi2ELi4EEEv": (8, 1), "fp8_reduce_kernel": (4, 8), "rotary_qkv_kernelIDF16bDF16b": (8, 2),
            "quantize_fp8_rows_kernel": (4, 5), "quantize_fp8_weight_kernel": (4, 6), "ln_modulate_fp8_kernel": (1, 8)}


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
