"""What the kernels of the paged cache of 8-bit floating point work out from device arrays, on the CPU (tests/paged8_stub.cpp), under AddressSanitizer and
UndefinedBehaviorSanitizer.  Nothing here touches a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = os.environ.get("ROCM_CLANG", "/opt/rocm/llvm/bin/clang++")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++")
    exe = str(tmp_path_factory.mktemp("paged8_stub") / "paged8_stub")
    cmd = [CLANG, "-O1", "-g", "-std=c++20", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-unused-value", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", os.path.join(ROOT, "tests", "paged8_stub.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    if r.returncode != 0 and "sanitize" in r.stderr and "unsupported" in r.stderr:
        pytest.skip("this toolchain has no host sanitizers: " + r.stderr[-200:])
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


@pytest.mark.parametrize("scenario", ["join", "lookup", "rows"])
def test_on_the_cpu(program, scenario):
    r = subprocess.run([program, scenario], capture_output=True, text=True, timeout=600)
    if r.returncode != 0 and "ASan runtime does not come first" in r.stderr:
        pytest.skip(r.stderr[-300:])
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), (r.returncode, r.stdout[-2000:], r.stderr[-3000:])
