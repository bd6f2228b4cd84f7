"""The host code of the gated layers, lookups and orthogonalised updates on a HIP runtime
made of stubs (tests/heads_host_driver.cpp): what it refuses, which device it works on,
what a failed allocation leaves."""
import os
import shutil
import subprocess

import pytest

from paper_2011_12490_amd import build


def test_host_code_on_a_stub_runtime(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "heads_host")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "heads_host_driver.cpp"),
                    os.path.join(build.CSRC, "heads_api.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "heads host driver: 0 failure(s)" in r.stdout
