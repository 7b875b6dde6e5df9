"""The kernels that the sizes of the GPU tests of the product in 8 bits are meant for are the ones that the library picks."""
import os
import shutil
import subprocess

import pytest

import test_gpu_q8_paths as paths
from q8_cases import FEW_CHANNELS, FEW_ROWS, FEW_WIDTHS, RING, STEPS

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIBDIR = os.path.join(ROOT, "paper_2507_17301_amd")
LIB = os.path.join(LIBDIR, "libnmconv.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libnmconv.so not built (python -m paper_2507_17301_amd.build)")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan([(rows, k, channels, gated)]) -> [(shape, splits, steps of a part, steps)]"""
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        clang = shutil.which("amdclang++")
    if not clang:
        pytest.skip("no HIP-aware clang++ in this image")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    r = subprocess.run([clang, "-x", "hip", "--cuda-host-only", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(LIBDIR, "csrc"), "-I", "/opt/rocm/include", os.path.join(HERE, "q8_plan_print.cpp"),
                        "-x", "none", LIB, "-Wl,-rpath," + LIBDIR, "-o", exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

    def ask(sizes):
        r = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in sizes), capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        lines = [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]
        assert len(lines) == len(sizes)
        return lines
    return ask


def _sizes(test):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == "rows,k,n")


def test_undivided_tiles_go_round_their_stages(plan):
    for shape, sizes in RING.items():
        for gated in (0, 1):
            for (rows, k, n), got in zip(sizes, plan([(rows, k, n, gated) for rows, k, n in sizes])):
                assert got == (shape, 1, got[2], STEPS[k]), (rows, k, n, gated, got)
                assert STEPS[k] == (k + 127) // 128 and STEPS[k] >= 7


def test_sizes_for_each_shape_take_it_whole_and_divided(plan):
    whole, divided = set(), set()
    for (rows, k, n), (shape, splits, per, steps) in zip(sizes := _sizes(paths.test_each_shape_of_tile), plan([(*s, 0) for s in sizes])):
        (divided if splits > 1 else whole).add(shape)
        assert splits == 1 or (splits - 1) * per < steps <= splits * per
    assert whole == set(range(7)) and divided >= {0, 1, 2, 3, 4, 5, 6}, (whole, divided)


def test_up_to_64_rows_take_the_few_row_kernels(plan):
    sizes = [(rows, k, n, 0) for rows in FEW_ROWS for k in FEW_WIDTHS for n in FEW_CHANNELS]
    assert all(p[0] == -1 and p[1] == 1 for p in plan(sizes))
    assert [p[0] >= 0 for p in plan([(64, 4096, 4096, 0), (65, 4096, 4096, 0)])] == [False, True]
