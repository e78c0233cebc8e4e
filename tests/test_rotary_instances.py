"""Which forms of the rotation there are: what a norm needs is not asked of rows without one."""
from tests.test_kernel_resources import _all, kernels  # noqa: F401

NO_NORM = 0


def test_rows_without_a_norm_have_a_form_of_their_own(kernels):  # noqa: F811
    """Every width of chunks, one slot a lane, every pair of types (t: bfloat16, f: single precision; 16-byte chunks of bfloat16 alone)."""
    for types in ("tt", "tf", "ft", "ff"):
        for width in (1, 2, 4) + ((8,) if types == "tt" else ()):
            _all(kernels, "rotate_kernelI%sLi%dELi1ELNS0_8NormFormE%dE" % (types, width, NO_NORM))
