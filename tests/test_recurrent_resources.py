"""What the launches of the recurrent operators rest on, read from the kernel descriptors hipcc
writes for gfx950: three workgroups of a segment's scan share a compute unit, two of the scan of
whole sequences and of the gradients; no kernel but these scans uses scratch, and they little;
copies of beam states stay in registers. No GPU is needed."""
import re

import pytest

from test_kernel_resources import REGS_PER_LANE, _kernel_descriptors

SOURCES = ("scan.hip", "scan_backward.hip", "scan_step.hip", "conv.hip", "beam.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(kernel, its template arguments as they are mangled): descriptor}"""
    found = {}
    for source in SOURCES:
        for name, f in _kernel_descriptors(tmp_path_factory, source).items():
            m = re.search(r"\d(k_[a-z_]+?)(I\w+E)?E[vN]", name)
            assert m, name
            found[(m[1], m[2] or "")] = f
    return found


def _waves(f):
    """Waves that a SIMD's registers hold."""
    return REGS_PER_LANE // (-(-f["next_free_vgpr"] // 8) * 8)


def test_all_are_here(kernels):
    names = {k for k, _ in kernels}
    assert names == {"k_scan", "k_scan_prefix", "k_scan_parts", "k_scan_backward", "k_scan_low",
                     "k_scan_params", "k_scan_step", "k_conv", "k_conv_backward", "k_conv_sums",
                     "k_conv_step", "k_beam_pieces", "k_beam_merge", "k_beam_reorder"}
    assert sum(k == "k_conv" for k, _ in kernels) == 14   # two types, two to eight taps


def test_workgroups_share_a_unit(kernels):
    for (name, args), f in kernels.items():
        if name in ("k_scan", "k_scan_parts", "k_scan_backward"):   # workgroups of eight waves
            want = 6 if name == "k_scan" and args.endswith("Lb0EE") else 4
            assert _waves(f) >= want, (name, args, f["next_free_vgpr"])


def test_scratch(kernels):
    for (name, args), f in kernels.items():
        limit = 256 if name == "k_scan_backward" else 64 if name == "k_scan" else 0
        assert f["private_segment_fixed_size"] <= limit, (name, args, f)


def test_copies_stay_in_registers(kernels):
    assert kernels["k_beam_reorder", ""]["group_segment_fixed_size"] == 0


def test_only_the_gated_fp32_gradients_use_scratch(kernels):
    """And no more of it than when they were measured, 48 bytes a lane. Others that lost theirs
    gained by it (bf16 gradients: 132 bytes, 585 us with and 515 without at 4 x 4096 x 2048 x 16)."""
    allowed = {("k_scan_backward", "IfLb1EE"): 48}
    for at, f in kernels.items():
        assert f["private_segment_fixed_size"] <= allowed.get(at, 0), (at, f)
