"""The feed-forward kernels keep what they hold in registers: hipcc's report of each file names no scratch memory."""
import os
import subprocess

import pytest

from paper_1704_07724_amd import build


@pytest.mark.parametrize("name", ["rmsnorm", "route", "w4_linear", "w4_skip", "w4_pack"])
def test_no_scratch(name):
    build.generate()
    r = subprocess.run([build.HIPCC, *build.DEVICE_FLAGS, "-Rpass-analysis=kernel-resource-usage", "--cuda-device-only", "-c",
                        os.path.join(build.CSRC, name + ".hip"), "-o", os.devnull], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr
    assert "Function Name" in r.stderr and build._spills(r.stderr) == []
