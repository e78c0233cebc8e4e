"""Scalar registers of the kernels of rotation and shared pages: what does not fit goes over lanes of vector registers, never over memory, and only where both kinds of tile are in one kernel."""
import pytest

from tests.test_kernel_resources import _all, kernels  # noqa: F401


@pytest.mark.parametrize("part", ["rotate_kernel", "append_rotated_kernel", "append_rotated_token_kernel", "share_plan_kernel", "share_join_kernel"])
def test_scalars_stay_where_they_are(kernels, part):  # noqa: F811
    for n, r in _all(kernels, part).items():
        assert r["sgpr_spill_count"] == 0, (n, r)


def test_rows_of_shared_pages_keep_most_of_them(kernels):  # noqa: F811
    """48 for heads of 128 and 36 for heads of 64, less than a lane each of one vector register (the attention over pages alone: 12 and 4)."""
    for n, r in _all(kernels, "share_rows_kernel").items():
        assert r["sgpr_spill_count"] <= 48 and r["private_segment_fixed_size"] == 0, (n, r)
