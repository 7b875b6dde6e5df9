"""What the library launches for a product in MX4, asked on the CPU."""
import os
import re
import shutil
import subprocess
from typing import NamedTuple

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
F32, BF16, MX4 = 0, 1, 4


class Launch(NamedTuple):
    name: str          # mx4_few_kernel or mx4_tile_kernel
    args: tuple        # its template's arguments
    workgroups: int
    threads: int
    each: int          # few rows: workgroups of a tile of rows; tiles: tiles of channels
    first: int         # few rows: the first tile of rows; tiles: the first workgroup

    @property
    def rows(self):
        """Rows of a tile."""
        return 16 * (self.args[0] if self.name == "mx4_few_kernel" else self.args[1])


def build(folder):
    """The program that prints the launches, or None where there is no compiler for it."""
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        clang = shutil.which("amdclang++")
    if not clang:
        return None
    exe = os.path.join(str(folder), "launches")
    # (host pass only: the device code's image is the one symbol that is missing, and nothing looks at it)
    r = subprocess.run([clang, "-x", "hip", "--cuda-host-only", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(ROOT, "paper_2507_17301_amd", "csrc"), "-I", "/opt/rocm/include",
                        os.path.join(ROOT, "paper_2507_17301_amd", "csrc", "nm_mx4_product.hip"), os.path.join(HERE, "mx4_launch_print.cpp"),
                        "-Wl,--unresolved-symbols=ignore-in-object-files", "-no-pie", "-o", exe],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]
    return exe


def launches(exe, sizes):
    """[(rows, experts (0: one matrix), channels, width, gated, out)] -> [[Launch]]"""
    r = subprocess.run([exe], input="".join("%d %d %d %d %d %d\n" % tuple(s) for s in sizes), capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "refused" not in r.stdout, r.stdout + r.stderr
    out, now = [], []
    for line in r.stdout.splitlines():
        if line == "end":
            out.append(now)
            now = []
        else:
            name, args, rest = re.fullmatch(r"(?:void)?(?:nm::)?(?:\(anonymous namespace\)::)?(\w+)<([^>]*)> (.*)", line).groups()
            values = tuple({"true": 1, "false": 0}.get(v) if v in ("true", "false") else int(v) for v in args.split(","))
            now.append(Launch(name, values, *(int(v) for v in rest.split())))
    assert len(out) == len(sizes)
    return out
