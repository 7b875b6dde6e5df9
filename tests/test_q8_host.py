"""The host side of the 8-bit operators, with no GPU: exported symbols, the binding's argument blocks, refusals, and a sanitizer
run of the C entry points with stand-ins for the HIP runtime and the launchers."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "nm_q8.h")
LIB = os.path.join(ROOT, "paper_2507_17301_amd", "libnmconv.so")
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libnmconv.so not built (python -m paper_2507_17301_amd.build)")


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(nm_[a-z0-9_]+)\s*\(", text)))


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "nm_q8.h"\nint main(void) { return (int)sizeof(nm_linear_q8_args_t) * 0; }\n')
    for cc in (["gcc", "-std=c99"], ["g++", "-x", "c++", "-std=c++11"]):
        r = subprocess.run(cc + ["-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr


@built
def test_library_exports_every_declared_symbol():
    names = _declared()
    assert {"nm_rmsnorm_q8", "nm_quantize_q8", "nm_dequantize_q8", "nm_q8_pack", "nm_linear_q8"} <= set(names)
    L = ctypes.CDLL(LIB)
    for name in names:
        assert hasattr(L, name), f"{name} declared in nm_q8.h but not exported"


@built
def test_the_bindings_blocks_have_the_headers_sizes():
    from paper_2507_17301_amd import binding as nm
    # (the sizes themselves are asserted in C, in sanitize/q8_host_san.cpp)
    assert (nm._ROWS_ARGS.size, nm._DEQUANTIZE_ARGS.size, nm._LINEAR_ARGS.size) == (128, 72, 120)
    text = open(HEADER).read()
    assert int(re.search(r"NM_Q8_MAX_WIDTH = (\d+)", text).group(1)) == nm.NM_Q8_MAX_WIDTH
    assert int(re.search(r"NM_Q8_FEW_ROWS = (\d+)", text).group(1)) == nm.NM_Q8_FEW_ROWS
    assert int(re.search(r"NM_I8 = (\d+)", text).group(1)) == nm.NM_I8


@built
def test_refusals_need_no_gpu():
    from paper_2507_17301_amd import binding as nm
    L = nm.lib()
    buf = ctypes.create_string_buffer(4096)
    at = ctypes.addressof(buf) // 16 * 16 + 16
    q, s, x = at, at + 1024, at + 2048
    assert L.nm_quantize_q8(x, nm.NM_I8, 2, 16, 16, q, 16, s, None) == nm.NM_ERR_ARG
    assert L.nm_quantize_q8(x, nm.NM_F32, 2, nm.NM_Q8_MAX_WIDTH + 1, 16, q, 16, s, None) == nm.NM_ERR_SHAPE
    assert L.nm_quantize_q8(x, nm.NM_F32, 2, 16, 16, x, 16, s, None) == nm.NM_ERR_ARG
    assert b"overlaps" in L.nm_last_error()
    assert L.nm_quantize_q8(None, nm.NM_F32, 0, 16, 16, None, 16, None, None) == nm.NM_OK
    assert L.nm_linear_q8(q, 2, 16, 16, s, None, None, None, 0, x, nm.NM_F32, 8, None, 0, None) == nm.NM_ERR_ARG
    assert b"null handle" in L.nm_last_error()
    for name in ("nm_rows_q8_args", "nm_dequantize_q8_args", "nm_linear_q8_args"):
        assert getattr(L, name)(None) == nm.NM_ERR_ARG
    # the older calls do not take the new element type
    assert L.nm_maxpool2d(x, nm.NM_I8, 1, 4, 4, 4, 2, 2, 0, q, None) == nm.NM_ERR_ARG


def test_host_layer_under_asan_ubsan(tmp_path):
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not os.path.exists(clang):
        clang = shutil.which("amdclang++")
    if not clang:
        pytest.skip("no HIP-aware clang++ in this image")
    exe = str(tmp_path / "q8_san")
    # host pass only: no device code, no HIP runtime library -- the driver file supplies both
    cmd = ([clang, "-x", "hip", "--cuda-host-only", "-std=c++17", "-D__HIP_PLATFORM_AMD__"] + SAN +
           ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2507_17301_amd", "csrc"), "-I", "/opt/rocm/include",
            os.path.join(ROOT, "paper_2507_17301_amd", "csrc", "nm_q8_api.hip"), os.path.join(ROOT, "tests", "sanitize", "q8_host_san.cpp"), "-o", exe])
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600, env=env)
    assert r.returncode == 0 and "sanitizer run: ok" in r.stdout, r.stdout[-4000:]
