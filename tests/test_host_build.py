"""The build's commands with HIPCC given as a path, through a link, or as a name that PATH finds."""
import os
import shutil

import pytest

from paper_2607_04031_amd import build


def _headers(cmd):
    dirs = [cmd[i + 1] for i, x in enumerate(cmd) if x == "-isystem"]
    assert all(os.path.isabs(d) for d in dirs), dirs
    return [d for d in dirs if os.path.exists(os.path.join(d, "hip", "hip_runtime.h"))]


@pytest.mark.parametrize("how", ["path", "name", "link"])
def test_the_extension_module_finds_hip(how, monkeypatch, tmp_path):
    real = shutil.which(build.HIPCC)
    if not real:
        pytest.skip("hipcc is not available")
    given = real
    if how == "name":
        monkeypatch.setenv("PATH", os.path.dirname(real) + os.pathsep + os.environ["PATH"])
        given = os.path.basename(real)
    elif how == "link":
        given = str(tmp_path / "hipcc")
        os.symlink(real, given)
    monkeypatch.setattr(build, "HIPCC", given)
    assert _headers(build.calls_command(str(tmp_path / "out.so")))
