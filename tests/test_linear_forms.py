"""Which kernels the heads' layers launch, without a GPU (tests/linear_forms_driver.cpp
runs the library's own choice and writes kernels down by name): the GPU tests' cases
reach every one, so that a rule that moves takes no kernel out of their sight."""
import os
import shutil
import subprocess

import pytest

import test_gpu_heads
import test_gpu_heads_forms as forms
from paper_2011_12490_amd import build


def call(name, bf16, rows, heads, fan_in, fan_out, pad, shift, *more):
    return " ".join(str(int(v)) if not isinstance(v, str) else v
                    for v in (name, bf16, rows, heads, fan_in, fan_out, pad, shift) + more)


def bits(outputs):
    return sum(1 << i for i, wanted in enumerate(outputs) if wanted)


def calls_of_the_tests():
    """test_gpu_heads' and test_gpu_heads_forms' calls of the layers."""
    calls = []
    for bf16 in (0, 1):
        for counts, tail, I, O, pad, shift in test_gpu_heads.LINEAR_CASES:
            at = (bf16, sum(counts) + tail, len(counts), I, O, pad, shift)
            calls.append(call("forward", *at))
            calls += [call("backward", *at, relu, outputs) for relu in (0, 1) for outputs in (7, 6)]
        rows = (sum(forms.STREAM_ROWS[0]) + forms.STREAM_ROWS[1], len(forms.STREAM_ROWS[0]))
        calls += [call("forward", bf16, *rows, I, O, 0, 0) for I, O in forms.STREAM_FORWARD]
        calls += [call("backward", bf16, *rows, I, O, 0, 0, relu, outputs)
                  for I, O in forms.STREAM_BACKWARD for relu in (0, 1) for outputs in (7, 1)]
        calls += [call("backward", bf16, sum(counts) + tail, len(counts), I, O, 0, 0, relu, bits(outputs))
                  for counts, tail, I, O in forms.OUTPUT_CASES for relu in (0, 1) for outputs in forms.OUTPUTS]
    for counts, tail, I, O in forms.LARGE:
        at = (1, sum(counts) + tail, len(counts), I, O, 0, 0)
        calls += [call("forward", *at)] + [call("backward", *at, relu, 7) for relu in (0, 1)]
    return calls


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    """All kernels' names, and those that each of some calls launches."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    if not os.path.exists(os.path.join(build.BUILD, "kernels_linear.o")):
        build.build()
    exe = str(tmp_path_factory.mktemp("forms") / "linear_forms")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "linear_forms_driver.cpp"),
                    os.path.join(build.BUILD, "kernels_linear.o"), "-o", exe], check=True)

    def run(calls):
        r = subprocess.run([exe], input="\n".join(calls), capture_output=True, text=True, timeout=60, check=True)
        head, *per_call = r.stdout.split("call\n")
        assert len(per_call) == len(calls)
        names = [[line[4:] for line in part.splitlines() if line.startswith("ran ")] for part in per_call]
        return {line[4:] for line in head.splitlines() if line.startswith("has ")}, names

    return run


def test_the_gpu_tests_reach_every_kernel(launched):
    kernels, per_call = launched(calls_of_the_tests())
    assert len(kernels) > 100
    ran = {name for names in per_call for name in names}
    assert ran <= kernels
    assert not kernels - ran, "no test runs:\n" + "\n".join(sorted(kernels - ran))


def test_large_tiles_are_what_their_cases_say(launched):
    """The layer of the first and the rows' gradient of the second case of LARGE run in
    tiles of 256 x 256, with the rows' gradient in a launch of its own."""
    (counts, tail, I, O), (counts2, tail2, I2, O2) = forms.LARGE
    _, (layer, rows) = launched([call("forward", 1, sum(counts) + tail, len(counts), I, O, 0, 0),
                                 call("backward", 1, sum(counts2) + tail2, len(counts2), I2, O2, 0, 0, 0, 7)])
    large = [name for name in (layer[0], rows[0]) if "rows_kernel" in name and "Li256ELi256E" in name]
    assert len(layer) == 1 and len(large) == 2 and not any("gradients_kernel" in name for name in rows)
