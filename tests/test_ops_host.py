"""The training operators' host code on a HIP runtime made of stubs
(tests/ops_host_driver.cpp): what it refuses and which device it works on."""
import os
import shutil
import subprocess

import pytest

from paper_2011_12490_amd import build


def test_host_code_on_a_stub_runtime(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "ops_host")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "ops_host_driver.cpp"),
                    os.path.join(build.CSRC, "ops_api.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "ops host driver: 0 failure(s)" in r.stdout
