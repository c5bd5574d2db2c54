"""The page allocator under AddressSanitizer and UndefinedBehaviorSanitizer: tests/host/pager_driver.cpp drives it with random
calls.  Host code, CPU only."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_15943_amd", "csrc")
OUT = os.path.join(ROOT, "_build", "sanitize")


def test_page_allocator_under_address_and_ub_sanitizers():
    cxx = "/opt/rocm/llvm/bin/clang++"
    if not os.path.exists(cxx):
        pytest.skip("ROCm clang not installed")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "pager_driver")
    cmd = [cxx, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-fno-omit-frame-pointer", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "host", "pager_driver.cpp"), os.path.join(CSRC, "pager.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="halt_on_error=1:detect_leaks=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout, r.stderr)
    assert r.returncode == 0 and "pager checks passed" in r.stdout, r.stderr
    assert "runtime error" not in r.stderr
