"""CPU check of how the attention over pages deals out its work (tests/dealing_check.cpp): every tile once, and every worker's part
within the work, also that of a worker for whom there is none."""
import os
import shutil
import subprocess

import pytest

from tests.test_paging import CSRC, ROCM_INCLUDE, ROOT


def test_dealing(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("needs g++ and the ROCm headers")
    exe = str(tmp_path / "dealing_check")
    subprocess.run([cxx, "-O1", "-g", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-std=c++17", "-D__HIP_PLATFORM_AMD__",
                    "-I", ROCM_INCLUDE, "-I", CSRC, os.path.join(ROOT, "tests", "dealing_check.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
