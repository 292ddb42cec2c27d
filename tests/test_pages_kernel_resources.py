"""Compile-time guard (CPU, no GPU) for the page calls' kernels, as tests/test_kernel_resources.py for the products."""
from tests.test_kernel_resources import test_no_scratch_spills_and_lds_fits as _check


def test_no_scratch_spills(tmp_path):
    _check("tl_pages.hip", tmp_path)
