"""How an optimizer of orthogonalised updates puts its matrices into launches
(tests/muon_groups_driver.cpp on a HIP runtime made of stubs): small ones of several shapes
together, large ones within their workspace."""
import os
import shutil
import subprocess

import pytest

from paper_2011_12490_amd import build


def test_matrices_in_launches(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "muon_groups")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "muon_groups_driver.cpp"),
                    os.path.join(build.CSRC, "heads_api.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "muon groups driver: 0 failure(s)" in r.stdout
