"""The host side of the paged operators (paged_abi.cpp) built with the host compiler's
AddressSanitizer and UndefinedBehaviorSanitizer over stubs of the launchers, and driven by the CPU
tests of its C ABI."""
import os
import shutil
import subprocess
import sys

import pytest

from test_host_sanitizers import CSRC, ROOT, _runtime


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_paged_abi_under_asan_and_ubsan(tmp_path):
    asan = _runtime("libasan.so")
    if asan is None:
        pytest.skip("no AddressSanitizer runtime")
    lib = tmp_path / "libaatc_sanitized.so"
    stub = os.path.join(ROOT, "tests", "host_stub")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           *(os.path.join(CSRC, f) for f in ("calibrate.cpp", "abi.cpp", "group_abi.cpp", "paged_abi.cpp")),
           os.path.join(stub, "launch_stub.cpp"), os.path.join(stub, "paged_stub.cpp"), "-o", str(lib)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    env = dict(os.environ, AATC_LIBRARY=str(lib), LD_PRELOAD=asan,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    run = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                          os.path.join(ROOT, "tests", "test_paged_cpu.py")],
                         capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    tail = (run.stdout + run.stderr)[-3000:]
    assert run.returncode == 0, tail
    assert "passed" in run.stdout and "ERROR: AddressSanitizer" not in tail
    assert "runtime error" not in tail
