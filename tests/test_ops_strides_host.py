"""Strides at the ends of their range (no GPU): what the overlap check adds up
must not wrap around.  Run under the sanitizers too, which name an overflow."""

import ctypes
import os
import subprocess
import sys

import pytest

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import P, built  # noqa: F401  (builds the library)

BIG = 1 << 40


def _rope(tokens, heads, x, y):
    d = ops.RopeDesc(heads, 64, 1, (ctypes.c_int32 * 4)(64), 0, S.BF16)
    return ops.lib().pulse_rope(d, tokens, 0, x, P, P, y, None)


@pytest.mark.parametrize("tokens,heads,ts,hs", [
    # both strides alike, so token 1 of head 0 is head 1 of token 0; the
    # tokens' extent passes 2^63 and 2^64
    (1 << 24, 2, BIG, BIG), (1 << 23, 2, BIG, BIG), ((1 << 24) - 1, 2, BIG, BIG),
    # distinct elements, but no memory holds them
    (1 << 24, 1, BIG, 64), (1 << 24, 1024, BIG, 64), (1 << 16, 1024, 64, BIG),
])
def test_extents_that_no_memory_holds(tokens, heads, ts, hs):
    far, near = ops.Heads(P, ts, hs), ops.Heads(P, heads * 64, 64)
    for x, y in ((near, far), (far, near), (far, far)):
        assert _rope(tokens, heads, x, y) == S.E_INVALID_ARG
        assert S.lib().pulse_last_error()


def test_attention_refuses_them_too():
    d = ops.AttnDesc(1 << 24, 1 << 24, 2, 1, 64, 0.125, 0.0, S.BF16)
    near, far, k = ops.Heads(P, 128, 64), ops.Heads(P, BIG, BIG), ops.Heads(P, 64, 64)
    L = ops.lib()
    for q, o in ((far, near), (near, far)):
        assert L.pulse_attn_forward(d, q, k, k, P, None, o, P, None, P, BIG,
                                    None) == S.E_INVALID_ARG


def test_strides_under_asan_and_ubsan():
    if "PULSE_STAGE_LIB" in os.environ:
        pytest.skip("runs the tests of this file in the sanitizers' build")
    from paper_2606_19163_amd import build as B
    env = dict(os.environ)
    env.update({"PULSE_STAGE_LIB": B.build_asan(), "LD_PRELOAD": B.asan_runtime(),
                "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
                "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1",
                "HIP_VISIBLE_DEVICES": ""})
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
           os.path.abspath(__file__)]
    r = subprocess.run(cmd, env=env, capture_output=True, text=True, timeout=900)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in tail and "runtime error" not in tail, tail
