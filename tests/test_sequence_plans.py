"""What the sequence operators' plans decide, checked on the CPU under AddressSanitizer and
UndefinedBehaviorSanitizer: csrc_seq/seq_host.h, compiled by g++ as host code only and driven by
tests/sanitize/seq_plan_harness.cpp."""
import os
import shutil
import subprocess

import pytest

from tests.test_sequence_sanitizers import ROOT, SAN


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans_under_sanitizers(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = tmp_path / "seq_plan_harness"
    csrc = [os.path.join(ROOT, "paper_2408_00280_amd", d) for d in ("csrc", "csrc_seq")]
    include = [f for d in (os.path.join(rocm, "include"), os.path.join(ROOT, "include"), *csrc) for f in ("-I", d)]
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", *include,
                    os.path.join(ROOT, "tests", "sanitize", "seq_plan_harness.cpp"), "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "all checks passed" in r.stdout
