"""Arrays that share memory: the host code of the gated layers, lookups and orthogonalised
matrices against a map of bytes, and what its entry points refuse
(tests/heads_arrays_driver.cpp, on launches that run nothing)."""
import os
import shutil
import subprocess

import pytest

from paper_2011_12490_amd import build


def test_arrays_that_share_memory(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "heads_arrays")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Wno-unused-function", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "heads_arrays_driver.cpp"),
                    os.path.join(build.CSRC, "heads_api.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "heads arrays driver: 0 failure(s)" in r.stdout
