"""Compile-time guard (CPU, no GPU) for the serving kernels, as tests/test_kernel_resources.py for the products: no scratch
(private memory) spills, and static LDS within gfx950's 160 KB."""
import pytest

from tests.test_kernel_resources import test_no_scratch_spills_and_lds_fits as _check


@pytest.mark.parametrize("src", ["tl_kv.hip", "tl_attn.hip", "tl_attn_wide.hip", "tl_verify.hip"])
def test_no_scratch_spills(src, tmp_path):
    _check(src, tmp_path)
