"""The 4-bit cache's host code under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): its source and the shared host plumbing
are compiled as host code and linked with tests/kv4_host_check.cpp."""
import os
import subprocess

from test_abi_sanitized_cpu import CSRC, HOST_CXX, INCLUDE, ROCM, ROOT, SAN, _hipcc, _run


def test_host_code_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "kv4_host_check")
    kv4 = os.path.join(CSRC, "kv4")
    _run([_hipcc(), "-O1", "-g", "-std=c++17", "-I", INCLUDE, "-I", CSRC, "-I", kv4, *SAN,
          *HOST_CXX, os.path.join(kv4, "mg_kv4.cpp"), os.path.join(CSRC, "host_runtime.cpp"),
          os.path.join(ROOT, "tests", "kv4_host_check.cpp"), "-o", exe, "-L",
          os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib")])
    env = dict(os.environ)
    env["ASAN_OPTIONS"] = "detect_leaks=1:abort_on_error=0:halt_on_error=1"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-6000:]
    assert "kv4 host checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
