"""What a workgroup of the attention kernels knows of its piece of work has a value from the start (csrc/tl_attn_device.h): not
every path sets every member before the others read it.  A constant of such a type needs one.  Checked by the compiler, not run."""
import os
import subprocess

import pytest

from paper_2607_04031_amd import build

SOURCE = """
#include <hip/hip_runtime.h>
#include "tl_attn_device.h"
constexpr tl::AttnPiece piece;
static_assert(piece.s.before == 0 && piece.slot == 0 && !piece.whole, "");
"""


def test_pieces_have_values_from_the_start(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc is not available")
    src = tmp_path / "values.hip"
    src.write_text(SOURCE)
    cmd = [build.HIPCC, *[f for f in build.FLAGS if f != "-fPIC"], "-I" + build.CSRC, "--cuda-device-only", "-fsyntax-only", str(src)]
    out = subprocess.run(cmd, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
