"""The feed-forward kernels keep what they hold in registers: hipcc's report of each file names no scratch memory."""
import glob
import os
import re
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


def test_assembly_names_the_registers_that_it_writes():
    """m0 is the compiler's too: an asm that sets it says so."""
    seen = 0
    for path in glob.glob(os.path.join(build.CSRC, "*.h*")):
        with open(path) as f:
            text = f.read()
        for statement in re.findall(r"\basm\b[^;]*?\((.*?)\);", text, re.S):
            written = re.search(r"\bs_\w+ (m0|vcc|exec|s\d+|s\[)", statement)
            if written:
                seen += 1
                assert '"%s"' % written.group(1) in statement.split(":")[-1], (path, statement)
    assert seen > 0
