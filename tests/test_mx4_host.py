"""The host side of the operators in MX4 and of those for experts, with no GPU: exported symbols, the binding's argument blocks,
refusals, and a sanitizer run of the C entry points with stand-ins for the HIP runtime and the launchers."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = {name: os.path.join(ROOT, "include", name) for name in ("nm_mx4.h", "nm_experts.h")}
LIB = os.path.join(ROOT, "paper_2507_17301_amd", "libnmconv.so")
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libnmconv.so not built (python -m paper_2507_17301_amd.build)")


def _text():
    return re.sub(r"/\*.*?\*/", "", "".join(open(h).read() for h in HEADERS.values()), flags=re.S)


@pytest.mark.parametrize("header,block", [("nm_mx4.h", "nm_product_mx4_args_t"), ("nm_experts.h", "nm_route_args_t")])
def test_headers_are_plain_c(tmp_path, header, block):
    src = tmp_path / "h.c"
    src.write_text(f'#include "{header}"\nint main(void) {{ return (int)sizeof({block}) * 0; }}\n')
    for cc in (["gcc", "-std=c99"], ["g++", "-x", "c++", "-std=c++11"]):
        r = subprocess.run(cc + ["-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr


@built
def test_library_exports_every_declared_symbol():
    names = sorted(set(re.findall(r"\b(nm_[a-z0-9_]+)\s*\(", _text())))
    assert {"nm_rmsnorm_mx4", "nm_quantize_mx4", "nm_dequantize_mx4", "nm_mx4_pack", "nm_linear_mx4", "nm_experts_mx4", "nm_route", "nm_combine"} <= set(names)
    L = ctypes.CDLL(LIB)
    for name in names:
        assert hasattr(L, name), f"{name} declared but not exported"


@built
def test_the_bindings_blocks_have_the_headers_sizes():
    from paper_2507_17301_amd import binding as nm
    # (the sizes themselves are asserted in C, in sanitize/mx4_host_san.cpp)
    blocks = (nm._ROWS4_ARGS, nm._DEQUANTIZE4_ARGS, nm._PRODUCT4_ARGS, nm._ROUTE_ARGS, nm._COMBINE_ARGS)
    assert tuple(b.size for b in blocks) == (136, 80, 152, 120, 120)
    for name in ("NM_MX4", "NM_ROUTE_MAX_EXPERTS", "NM_ROUTE_MAX_CHOICES", "NM_ROUTE_ONE_LAUNCH"):
        assert int(re.search(name + r" = (\d+)", _text()).group(1)) == getattr(nm, name)


@built
def test_refusals_need_no_gpu():
    from paper_2507_17301_amd import binding as nm
    L = nm.lib()
    buf = ctypes.create_string_buffer(4096)
    at = ctypes.addressof(buf) // 16 * 16 + 16
    x, q, s = at, at + 1024, at + 2048
    assert L.nm_quantize_mx4(x, nm.NM_MX4, 2, 64, 64, q, 32, s, 2, None) == nm.NM_ERR_ARG
    assert L.nm_quantize_mx4(x, nm.NM_F32, 2, 64, 64, q + 8, 32, s, 2, None) == nm.NM_ERR_ARG
    assert b"16 bytes" in L.nm_last_error()
    assert L.nm_quantize_mx4(x, nm.NM_F32, 2, 64, 64, x, 32, s, 2, None) == nm.NM_ERR_ARG
    assert b"overlaps" in L.nm_last_error()
    assert L.nm_quantize_mx4(x, nm.NM_F32, 2, nm.NM_Q8_MAX_WIDTH + 1, 64, q, 32, s, 2, None) == nm.NM_ERR_SHAPE
    assert L.nm_quantize_mx4(None, nm.NM_F32, 0, 64, 64, None, 32, None, 2, None) == nm.NM_OK
    assert L.nm_linear_mx4(q, 32, s, 2, 2, 64, None, None, None, 0, x, nm.NM_F32, 8, None, 0, None) == nm.NM_ERR_ARG
    assert b"null handle" in L.nm_last_error()
    assert L.nm_route(x, nm.NM_F32, 2, 8, 8, 9, 1, q, q + 64, q + 128, q + 256, q + 512, None, 0, None) == nm.NM_ERR_ARG
    assert L.nm_combine(x, nm.NM_F32, 2, 8, q, q + 64, 2, 0, 8, None, 0, s, nm.NM_F32, 8, None) == nm.NM_ERR_ARG
    for name in ("nm_rows_mx4_args", "nm_dequantize_mx4_args", "nm_product_mx4_args", "nm_route_args", "nm_combine_args"):
        assert getattr(L, name)(None) == nm.NM_ERR_ARG
    # the older calls do not take the new element type
    assert L.nm_maxpool2d(x, nm.NM_MX4, 1, 4, 4, 4, 2, 2, 0, q, None) == nm.NM_ERR_ARG
    assert L.nm_quantize_q8(x, nm.NM_MX4, 2, 16, 16, q, 16, s, None) == nm.NM_ERR_ARG


def test_host_layer_under_asan_ubsan(tmp_path):
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        clang = shutil.which("amdclang++")
    if not clang:
        pytest.skip("no HIP-aware clang++ in this image")
    exe = str(tmp_path / "mx4_san")
    # host pass only: no device code, no HIP runtime library -- the driver file supplies both
    cmd = ([clang, "-x", "hip", "--cuda-host-only", "-std=c++17", "-D__HIP_PLATFORM_AMD__"] + SAN +
           ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2507_17301_amd", "csrc"), "-I", "/opt/rocm/include",
            os.path.join(ROOT, "paper_2507_17301_amd", "csrc", "nm_mx4_api.hip"), os.path.join(ROOT, "tests", "sanitize", "mx4_host_san.cpp"), "-o", exe])
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600, env=env)
    assert r.returncode == 0 and "sanitizer run: ok" in r.stdout, r.stdout[-4000:]
