"""Forks, cuts and read-back over a fake device (tests/moves_stub.hip), the host side under AddressSanitizer and UndefinedBehaviorSanitizer: page lists,
allocator, launches that fail, the sizes of launches.  Nothing here touches a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_18610_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SAN = ["-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("moves_stub")
    exe = str(at / "moves_stub")
    arch_host = [a for f in SAN for a in ("-Xarch_host", f)]
    base = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include"), "-x", "hip", "-Xclang", "-target-feature",
            "-Xclang", "-packed-fp32-ops", "-Wno-unused-value", *arch_host]
    steps = [base + ["-c", os.path.join(CSRC, "kvq_host.cpp"), "-o", str(at / "host.o")],
             base + ["-c", os.path.join(ROOT, "tests", "moves_stub.hip"), "-o", str(at / "stub.o")],
             # (no HIP library: what the host code needs of it is in the program)
             [HIPCC, "-no-hip-rt", "--offload-arch=gfx950", *SAN, str(at / "stub.o"), str(at / "host.o"), "-o", exe]]
    for cmd in steps:
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
        if r.returncode != 0 and "sanitize" in r.stderr and "unsupported" in r.stderr:
            pytest.skip("this toolchain has no host sanitizers: " + r.stderr[-200:])
        assert r.returncode == 0, r.stderr[-3000:]
    return exe


@pytest.mark.parametrize("scenario", ["random_calls", "random_calls_without_a_device", "many_units"])
def test_moves_over_a_fake_device(program, scenario):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([program, scenario], capture_output=True, text=True, timeout=600, env=env)
    if r.returncode == 77 or (r.returncode != 0 and "ASan runtime does not come first" in r.stderr):
        pytest.skip((r.stdout + r.stderr)[-300:])
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), (r.returncode, r.stdout[-2000:], r.stderr[-3000:])
