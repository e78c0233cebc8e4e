"""Registers of the cache's and the attention's kernels as built (the notes of their code objects)."""
import pytest

from tests.test_kernel_resources import _all, kernels  # noqa: F401


@pytest.mark.parametrize("part", ["cache_append_kernel", "cache_append_token_kernel", "cache_read_kernel", "cache_compact_kernel", "cache_copy_kernel",
                                  "few_rows_kernel", "page_rows_kernel", "join_rows_kernel", "tile_rows_kernelILi64E", "tile_rows_kernelILi128ELNS0_10TileSourceE0E"])
def test_no_scratch(kernels, part):  # noqa: F811
    for n, r in _all(kernels, part).items():
        assert r["vgpr_spill_count"] == r["private_segment_fixed_size"] == 0, (n, r)


def test_rows_over_keys_keep_two_wavefronts_a_simd(kernels):  # noqa: F811
    for part in ("few_rows_kernel", "page_rows_kernel", "tile_rows_kernel"):
        for n, r in _all(kernels, part).items():
            assert r["vgpr_count"] <= 256, (n, r)
