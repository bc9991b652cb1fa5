"""Host code of the layer operators under sanitizers (no GPU needed): the division constants
that the kernels use, and every host rejection path of include/olive_layers.h."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36246_amd", "csrc")
OBJ_DIR = os.path.join(ROOT, "paper_2609_36246_amd", "_build")
HIPCC = "/opt/rocm/bin/hipcc"
CLANG = "/opt/rocm/llvm/bin/clang"
INC = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
# Each sanitizer flag applies to host code only.
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=all"]

pytestmark = pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)),
                                reason="ROCm compilers not found")


def test_division(tmp_path):
    exe = str(tmp_path / "division")
    subprocess.run([CLANG + "++", "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__",
                    "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I/opt/rocm/include"] + INC +
                   [os.path.join(ROOT, "tests", "division_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


def test_rejections_under_asan_and_ubsan(tmp_path):
    from paper_2609_36246_amd import build
    others = [os.path.join(OBJ_DIR, s.replace(".hip", ".o")) for s in build.SOURCES if s != "layers_abi.hip"]
    if not all(os.path.exists(o) for o in others):
        build.build()
    abi, drv, exe = (str(tmp_path / n) for n in ("abi.o", "drv.o", "check"))
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC"] + SAN + INC +
                   ["-c", os.path.join(CSRC, "layers_abi.hip"), "-o", abi], check=True)
    subprocess.run([CLANG, "-O1", "-g", "-std=c11"] + SAN[1::2] + INC +
                   ["-c", os.path.join(ROOT, "tests", "layers_host_check.c"), "-o", drv], check=True)
    subprocess.run([HIPCC, "--offload-arch=gfx950"] + SAN + ["-o", exe, drv, abi] + others, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
