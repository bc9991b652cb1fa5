"""Index arithmetic of the layer operators at the ends of their documented ranges, on the host
under the undefined-behaviour sanitizer (no GPU needed)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG), reason="ROCm compilers not found")


def test_steps_and_grids(tmp_path):
    exe = str(tmp_path / "ranges")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2609_36246_amd", "csrc"), os.path.join(ROOT, "tests", "range_check.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr
