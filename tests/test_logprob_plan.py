"""The plans of the log probabilities: parts that cover a row, within the limits that
the kernels' words and LDS set, in no more scratch than is reported
(tests/logprob_plan_driver.cpp, host code)."""
import os
import shutil
import subprocess

import pytest

from paper_2510_26843_amd import build


@pytest.mark.skipif(not shutil.which("g++"), reason="no g++")
def test_scratch_holds_every_plan(tmp_path):
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I" + build.CSRC,
                    os.path.join(os.path.dirname(__file__), "logprob_plan_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "enough\n", r.stdout
