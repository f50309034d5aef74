"""The host side of drawn children, of the verification of trees and of adapted projections (csrc/api.cpp, csrc/marshal_sample.cpp) under AddressSanitizer
and UndefinedBehaviorSanitizer: the libraries of tests/sanitize_host.py, driven by these operators' host tests (no GPU involved)."""
import glob
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = ("test_sampling.py", "test_tree_verify.py", "test_adapters.py", "test_sampled_drafting.py")


def test_host_code_of_the_operators_is_clean_under_address_and_ub_sanitizers(tmp_path):
    if os.environ.get("MAMBA_HIP_LIB"):
        pytest.skip("already inside the sanitizer run")
    if not glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"):
        pytest.skip("no shared AddressSanitizer runtime in this image")
    import sanitize_host
    hip_lib, marshal, oracle_lib = sanitize_host.build(str(tmp_path))
    cxx = subprocess.check_output([os.environ.get("CXX", "g++"), "-print-file-name=libstdc++.so.6"], text=True).strip()
    env = dict(os.environ, MAMBA_HIP_LIB=hip_lib, MAMBA_HIP_MARSHAL=marshal, MAMBA_ORACLE_LIB=oracle_lib,
               LD_PRELOAD=":".join([sanitize_host.runtime(), cxx] + ([os.environ["LD_PRELOAD"]] if os.environ.get("LD_PRELOAD") else [])),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:exitcode=66:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1:exitcode=67")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-s", "-p", "no:cacheprovider", "-m", "not gpu"] + [os.path.join(ROOT, "tests", t) for t in TESTS],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-3000:]
    assert not any(k in out for k in ("ERROR: AddressSanitizer", "runtime error:", "SUMMARY: UndefinedBehaviorSanitizer")), out[-3000:]
    assert " passed" in r.stdout and " skipped" not in r.stdout, out[-1000:]
