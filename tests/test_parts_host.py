"""How the attention on bf16 pages finds the lengths of its parts (csrc/part_length.h), under UndefinedBehaviorSanitizer:
tests/host/parts_driver.cpp.  Host code, CPU only."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_15943_amd", "csrc")
OUT = os.path.join(ROOT, "_build", "sanitize")


def test_part_lengths_under_the_ub_sanitizer():
    cxx = "/opt/rocm/llvm/bin/clang++"
    if not os.path.exists(cxx):
        pytest.skip("ROCm clang not installed")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "parts_driver")
    cmd = [cxx, "-O1", "-g", "-std=c++17", "-fsanitize=undefined,float-cast-overflow", "-fno-sanitize-recover=all",
           "-I", CSRC, os.path.join(ROOT, "tests", "host", "parts_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "parts checks passed" in r.stdout, r.stdout + r.stderr
