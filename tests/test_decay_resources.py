"""What the decayed attention's launches rest on, read from the kernel descriptors hipcc writes
for gfx950: two workgroups of a bf16 scan share a compute unit, at 256 columns only because the
second terms of the pair weights take the values' place; so do those of the sums; scans of 64
columns and one value tile fit four times. Scratch: in the scans that hold as many states as
their registers allow, and little. No GPU is needed."""
import re

import pytest

from test_kernel_resources import LDS_PER_CU, REGS_PER_LANE, _kernel_descriptors


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(kernel, type, columns, waves, value tiles, whole): descriptor}"""
    found = {}
    for name, f in _kernel_descriptors(tmp_path_factory, "decay.hip").items():
        m = re.search(r"k_decay_(scan|sums)I(DF16b|f)Li(\d+)ELi(\d+)ELi(\d+)ELb(\d)EE", name)
        if m:
            found[(m[1], "f32" if m[2] == "f" else "bf16", *map(int, m.groups()[2:]))] = f
        else:
            assert "k_decay_prefix" in name, name
    assert len(found) == 30
    return found


def _fit(f, waves):
    """Workgroups of `waves` waves that a compute unit's registers and LDS hold."""
    per_simd = REGS_PER_LANE // (-(-f["next_free_vgpr"] // 8) * 8)
    return min(4 * per_simd // waves, LDS_PER_CU // f["group_segment_fixed_size"])


def test_workgroups_share_a_unit(kernels):
    for (kernel, dtype, columns, waves, tiles, whole), f in kernels.items():
        want = 1
        if dtype == "bf16":
            want = 4 if kernel == "scan" and columns == 64 and tiles == 1 else 2
        assert _fit(f, waves) >= want, (kernel, dtype, columns, waves, tiles, whole, f)


def test_scratch(kernels):
    for (kernel, dtype, columns, waves, tiles, whole), f in kernels.items():
        full = kernel == "scan" and dtype == "bf16" and columns * tiles == 256
        limit = (128 if whole else 16) if full else 0
        assert f["private_segment_fixed_size"] <= limit, (kernel, dtype, columns, waves, tiles,
                                                          whole, f["private_segment_fixed_size"])
