"""CPU check of the paged cache's index arithmetic (tests/paging_check.cpp): where places lie, tables that name pages which the cache does
not have, which slots an append writes, and the scales of a cache in 8 bits."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2206_08720_amd", "csrc")
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")


def test_paging(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("needs g++ and the ROCm headers")
    exe = str(tmp_path / "paging_check")
    subprocess.run([cxx, "-O1", "-g", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-std=c++17", "-D__HIP_PLATFORM_AMD__",
                    "-I", ROCM_INCLUDE, "-I", CSRC, os.path.join(ROOT, "tests", "paging_check.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr
