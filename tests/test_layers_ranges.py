"""Index arithmetic of the layer operators at the ends of their documented ranges, on the host
under the undefined-behaviour sanitizer (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_36246_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not os.path.exists(CLANG), reason="ROCm compilers not found")
def test_steps_and_grids(tmp_path):
    exe = str(tmp_path / "ranges")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2609_36246_amd", "csrc"), os.path.join(ROOT, "tests", "range_check.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


@pytest.mark.parametrize("sizes", [[(1 << 63) - 1], [(1 << 63) - 16384], [1 << 45], [1 << 44, 1 << 44],
                                   [5, (1 << 63) - 1], [(1 << 63) - 1, (1 << 63) - 16384]])
def test_gradients_of_too_many_values(sizes):
    """Their chunks are counted without passing 64 bits, and refused before anything is allocated."""
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_36246_amd import build
        build.build()
    t = (L.olive_grad_tensor * len(sizes))(*[L.olive_grad_tensor(1 << 20, 1 << 20, n, L.OLIVE_F32, L.OLIVE_F32)
                                             for n in sizes])
    h = ctypes.c_void_p()
    assert L.load().olive_grad_clip_init(ctypes.byref(h), t, len(sizes), None) == L.OLIVE_E_SHAPE
    assert h.value is None
