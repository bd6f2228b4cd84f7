"""Which kernels the gated layers, the table lookups and the orthogonalised updates launch,
without a GPU (tests/more_forms_driver.cpp runs the library's own choice and writes
kernels down by name): the GPU tests' cases reach every one, so that a rule that moves
takes no kernel out of their sight."""
import os
import shutil
import subprocess

import pytest

import test_gpu_heads_gated as gated
import test_gpu_lookup as lookup
import test_gpu_muon as muon
from paper_2011_12490_amd import build

UNITS = ["kernels_gated", "kernels_gated_back", "kernels_lookup", "kernels_muon"]


def line(name, *numbers):
    return " ".join([name] + [str(int(n)) for n in numbers])


def calls_of_the_tests():
    calls = []
    for bf16 in (0, 1):
        for counts, tail, I, O, pad, shift in gated.CASES:
            at = (bf16, sum(counts) + tail, len(counts), I, O, pad, shift)
            calls += [line("gated", *at, keep) for keep in (0, 1)] + [line("backward", *at, outputs) for outputs in (6, 7)]
        for counts, tail, I, O in gated.MORE:
            at = (bf16, sum(counts) + tail, len(counts), I, O, 0, 0)
            calls += [line("gated", *at, 1)] + [line("backward", *at, outputs) for outputs in (6, 7)]
        for T, V, D, pad, shift, _ in lookup.CASES:
            calls += [line("lookup", bf16, T, V, D, pad, shift), line("gradient", bf16, T, V, D, pad, shift)]
        for K, O, I in muon.SHAPES:
            calls.append(line("matrices", 1 - bf16, K, O, I))
    return calls


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    """All kernels' names, and those that each of some calls launches."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    objects = [os.path.join(build.BUILD, unit + ".o") for unit in UNITS]
    if not all(os.path.exists(o) for o in objects):
        build.build()
    exe = str(tmp_path_factory.mktemp("forms") / "more_forms")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "include")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I" + rocm,
                    "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(build.ROOT, "tests", "more_forms_driver.cpp")] + objects + ["-o", exe], check=True)

    def run(calls):
        r = subprocess.run([exe], input="\n".join(calls), capture_output=True, text=True, timeout=60, check=True)
        head, *per_call = r.stdout.split("call\n")
        assert len(per_call) == len(calls)
        names = [[row[4:] for row in part.splitlines() if row.startswith("ran ")] for part in per_call]
        return {row[4:] for row in head.splitlines() if row.startswith("has ")}, names

    return run


def test_the_gpu_tests_reach_every_kernel(launched):
    kernels, per_call = launched(calls_of_the_tests())
    assert len(kernels) > 60
    ran = {name for names in per_call for name in names}
    assert ran <= kernels
    assert not kernels - ran, "no test runs:\n" + "\n".join(sorted(kernels - ran))


def test_launches_of_ordinary_calls(launched):
    """How many launches a call takes: what a small call's time is made of."""
    calls = [line("gated", 1, 16, 16, 64, 64, 0, 0, 1), line("backward", 1, 500, 4, 128, 128, 0, 0, 7),
             line("lookup", 0, 64, 500, 48, 0, 0), line("gradient", 0, 64, 500, 48, 0, 0), line("gradient", 0, 5000, 500, 48, 0, 0),
             line("gradient", 0, 50000, 500, 48, 0, 0), line("matrices", 1, 144, 128, 128), line("matrices", 1, 3, 300, 700)]
    _, names = launched(calls)
    assert [len(n) for n in names] == [1, 2, 1, 1, 3, 5, 1, 18]


def test_few_samples_of_few_rows_are_sorted(launched):
    """The gradient of up to 256 samples: one launch while their rows spread over many workgroups,
    sorted where a workgroup would go through them all one after the other."""
    sizes = [(T, V, D) for T in (1, 64, 96) for V in (1, 2, 9, 500) for D in (3, 48, 1024)] + [
        (256, 500, 48), (256, 500, 1024), (256, 20000, 8), (200, 100000, 64)]
    spread = len(sizes)
    sizes += [(T, V, D) for T in (128, 256) for V in (1, 2) for D in (3, 48, 256, 1024)] + [(256, 9, 48), (256, 50, 8)]
    for bf16 in (0, 1):
        _, names = launched([line("gradient", bf16, T, V, D, 0, 0) for T, V, D in sizes])
        for size, kernels in zip(sizes[:spread], names[:spread]):
            assert len(kernels) == 1 and "few_kernel" in kernels[0], size
        for size, kernels in zip(sizes[spread:], names[spread:]):
            assert len(kernels) > 1 and not any("few_kernel" in k for k in kernels), size


def test_lookups_that_the_caches_hold_stay_there(launched):
    """Results of whole lines go past the caches only from 256 MB on."""
    sizes = [(0, 65536, 512), (1, 65536, 512), (1, 262143, 512), (0, 1000, 64), (1, 262144, 512), (0, 131072, 512), (0, 1 << 20, 64)]
    kernels, names = launched([line("lookup", bf16, T, 1000, D, 0, 0) for bf16, T, D in sizes])
    past = {k for k in kernels if "lookup_kernel" in k and "Lb1E" in k}
    assert len(past) == 2
    assert [n[0] in past for n in names] == [False] * 4 + [True] * 3


def test_gated_layers_of_large_tiles(launched):
    """Tiles of 256 as the layers' rule takes them; of 256 to 512 deep ones where few of them are
    left over for the last round."""
    small = [(131072, 16, 256, 256), (65536, 8, 320, 512), (65536, 64, 320, 512), (131072, 16, 384, 384), (65536, 16, 448, 640),
             (4096, 8, 2048, 2048)]
    large = [(262139, 16, 256, 256), (131072, 16, 320, 512), (65536, 16, 768, 768), (16384, 8, 2048, 2048)]
    _, names = launched([line("gated", 1, *size, 0, 0, 1) for size in small + large])
    assert [len(n) for n in names] == [1] * 10
    assert ["Li256ELi256E" in n[0] for n in names] == [False] * 6 + [True] * 4, names
