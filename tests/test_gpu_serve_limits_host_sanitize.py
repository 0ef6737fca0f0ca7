"""Adapters at the ends of what a call may say, under AddressSanitizer + UndefinedBehaviorSanitizer (host code only).  Driver: tests/host_sanitize/serve_limits.cpp."""
import os
import subprocess

import pytest

EXE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_05035_amd", "serve_limits_hostsan")


@pytest.mark.gpu
def test_the_ends_of_what_a_call_may_say_under_host_sanitizers():
    if not os.path.exists(EXE):
        pytest.skip("host sanitizer target not built (python paper_2603_05035_amd/build.py --sanitize)")
    env = dict(os.environ)
    # the HIP runtime keeps allocations until exit and maps memory where the sanitizer's shadow gap would be
    env["ASAN_OPTIONS"] = "detect_leaks=0:protect_shadow_gap=0:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([EXE], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-4000:]
    assert "AddressSanitizer" not in r.stdout and "runtime error" not in r.stdout, r.stdout[-4000:]
    assert "all calls as promised" in r.stdout
