"""Every instance of the cache's and the attention's kernels keeps its vector registers out of scratch memory."""
import pytest

from tests.test_kernel_resources import _all, kernels  # noqa: F401


@pytest.mark.parametrize("part", ["cache_reserve_kernel", "cache_append_kernel", "cache_append_token_kernel", "cache_read_kernel", "cache_fork_kernel", "cache_copy_kernel",
                                  "cache_compact_plan_kernel", "cache_compact_kernel", "cache_free_kernel", "few_rows_kernel", "page_rows_kernel", "tile_rows_kernel",
                                  "join_rows_kernel"])
def test_no_instance_spills(kernels, part):  # noqa: F811
    for n, r in _all(kernels, part).items():
        assert r["vgpr_spill_count"] == r["private_segment_fixed_size"] == 0, (n, r)


def test_dense_rows_have_every_instance(kernels):  # noqa: F811
    """Heads of 64 and 128, rows straight into LDS and through registers."""
    assert len(_all(kernels, "tile_rows_kernel")) == 4
