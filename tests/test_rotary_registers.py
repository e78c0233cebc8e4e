"""Registers of the rotation's kernels and of those for sequences that share pages: none goes over scratch memory, and what has to be resident twice a compute unit is."""
import pytest

from tests.test_kernel_resources import _all, kernels  # noqa: F401


@pytest.mark.parametrize("part", ["rotate_kernel", "append_rotated_kernel", "append_rotated_token_kernel", "share_plan_kernel", "share_rows_kernel", "share_join_kernel"])
def test_no_instance_spills(kernels, part):  # noqa: F811
    for n, r in _all(kernels, part).items():
        assert r["vgpr_spill_count"] == r["private_segment_fixed_size"] == 0, (n, r)


def test_two_workgroups_a_compute_unit(kernels):  # noqa: F811
    """Four wavefronts each, 512 registers a SIMD: 256 for a wavefront."""
    for n, r in _all(kernels, "share_rows_kernel").items():
        assert r["vgpr_count"] <= 256, (n, r)


def test_rows_by_wide_chunks_keep_three_wavefronts_a_simd(kernels):  # noqa: F811
    """16 bytes a chunk, two slots of pairs a lane (one register more than 168 is a wavefront less)."""
    for part in ("rotate_kernelIttLi8ELi1E", "rotate_kernelIffLi4ELi1E"):
        for n, r in _all(kernels, part).items():
            assert r["vgpr_count"] <= 168, (n, r)
