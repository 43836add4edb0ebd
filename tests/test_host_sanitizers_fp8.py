"""Host-side memory and undefined-behaviour checks of the 8-bit entry points:
the library's sources built for the host as for the other entry points, linked
with a driver of their own that also holds every launch against the device's
limits (grid and workgroup sizes)."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "host_sanitize"))


@pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="hipcc is needed to compile the library's host code")
def test_fp8_abi_under_address_and_ub_sanitizers(tmp_path):
    import build as host_build
    host_build.build(str(tmp_path))
    clang = os.path.join("/opt/rocm/llvm/bin", "clang++")
    san = ["-fsanitize=address", "-fsanitize=undefined"]
    obj, exe = str(tmp_path / "driver_fp8.o"), str(tmp_path / "fp8_sanitized")
    subprocess.run([clang, "-O1", "-g", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *san, "-fno-sanitize-recover=all",
                    "-I", "/opt/rocm/include", "-I", host_build.INCLUDE, "-c",
                    os.path.join(HERE, "host_sanitize", "driver_fp8.cpp"), "-o", obj], check=True)
    rest = [o for o in glob.glob(str(tmp_path / "*.o")) if os.path.basename(o) not in ("driver.o", "driver_fp8.o")]
    subprocess.run([clang, *san, obj, *rest, "-Wl,--wrap=hipLaunchKernel", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="abort_on_error=1:detect_leaks=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "checks passed" in r.stdout
    assert "runtime error" not in out and "ERROR: AddressSanitizer" not in out
