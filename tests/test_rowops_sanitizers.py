"""The host tests of the row operators again, against the build
whose host C++ carries AddressSanitizer and UndefinedBehaviorSanitizer.  CPU
only: nothing is launched."""

import os
import subprocess
import sys

from test_host_sanitizers import ROOT


def test_row_operator_host_tests_under_asan_and_ubsan():
    sys.path.insert(0, ROOT)
    from paper_2606_19163_amd import build as B
    env = dict(os.environ)
    env.update({
        "PULSE_STAGE_LIB": B.build_asan(),
        "LD_PRELOAD": B.asan_runtime(),
        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
        "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1",
        "HIP_VISIBLE_DEVICES": "",
    })
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
           os.path.join(ROOT, "tests", "test_rowops_host.py")]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in tail and "runtime error" not in tail, tail
