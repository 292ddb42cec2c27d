"""wait_for_lds_loads (csrc/tl_attn_device.h) stands between loads that write LDS past the registers and the reads of what they
wrote: the compiler must not take a value read before it for the one after it.  Compiled for gfx950, not run."""
import os
import re
import subprocess

import pytest

from paper_2607_04031_amd import build

SOURCE = """
#include <hip/hip_runtime.h>
#include "tl_attn_device.h"
__global__ void before_and_after(unsigned* out) {
    __shared__ unsigned s[64];
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("; loads into s" :: "v"(s) : "memory");
    const unsigned a = s[threadIdx.x];
    tl::wait_for_lds_loads();
    const unsigned b = s[threadIdx.x];
    out[threadIdx.x] = a * 3 + b;
}
"""


def test_reads_of_lds_stay_behind_the_wait(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc is not available")
    src = tmp_path / "order.hip"
    src.write_text(SOURCE)
    cmd = [build.HIPCC, *[f for f in build.FLAGS if f != "-fPIC"], "-I" + build.CSRC, "--cuda-device-only", "-S", str(src), "-o", str(tmp_path / "order.s")]
    subprocess.run(cmd, check=True, capture_output=True)
    text = (tmp_path / "order.s").read_text()
    code = text[text.index("; loads into s"):text.index("s_endpgm")]
    reads = [m.start() for m in re.finditer(r"\bds_read_b32", code)]
    waits = [m.start() for m in re.finditer(r"s_waitcnt vmcnt\(0\)", code)]
    assert len(reads) == 2, code
    assert any(reads[0] < w < reads[1] for w in waits), code
