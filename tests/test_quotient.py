"""The paged attention's division by the heads of a group (tests/quotient_driver.cpp,
host code): with 4092 heads to one kv head a reciprocal of 32 bits alone takes the
last head of token 256 for one of the next token."""
import os
import shutil
import subprocess

import pytest

from paper_2510_26843_amd import build


@pytest.mark.skipif(not shutil.which(build.HIPCC), reason="no hipcc")
def test_every_group_size(tmp_path):
    exe = str(tmp_path / "driver")
    subprocess.run([build.HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O2", "-I" + build.CSRC, "-I" + build.INCLUDE,
                    os.path.join(os.path.dirname(__file__), "quotient_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "exact\n", r.stdout
