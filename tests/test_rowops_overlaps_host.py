"""Overlaps that the row operators refuse before anything is enqueued: far inside large
kept rows.  CPU only; pointers are addresses that nothing reads."""

import ctypes

import pytest

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import built  # noqa: F401  (builds the library)

R = ops.Rows
C, T = 65536, 1 << 20  # 66 GiB of kept rows
KEPT, FREE = 1 << 44, 1 << 46
DESC = ops.KeepDesc(C, 1, S.BF16)


def _size(tokens=T):
    n = ctypes.c_size_t()
    assert ops.lib().pulse_keep_sizes(DESC, tokens, n) == S.OK
    return n.value


def _refused(status):
    assert status == S.E_INVALID_ARG and b"overlaps" in S.lib().pulse_last_error()


INSIDE = [0, 1 << 20, 1 << 31, (1 << 35) - 16, 1 << 35, 3 << 34, _size]


@pytest.mark.parametrize("at", INSIDE)
def test_large_kept_rows(at):
    """A tensor that begins anywhere in the kept rows, their last bytes included."""
    L, n = ops.lib(), _size()
    at = KEPT + (n // 16 * 16 - 16 if at is _size else at)
    x, free = R(at, C), R(FREE, C)
    _refused(L.pulse_keep_save(DESC, T, x, None, KEPT, n, None))
    _refused(L.pulse_keep_save(DESC, T, free, x, KEPT, n, None))
    _refused(L.pulse_keep_load(DESC, T, KEPT, n, x, None))
    _refused(L.pulse_keep_backward(DESC, T, free, KEPT, n, x, None, 0, None))
    _refused(L.pulse_keep_backward(DESC, T, x, FREE << 1, n, free, KEPT, n, None))
    _refused(L.pulse_keep_backward(DESC, T, free, KEPT, n, R(FREE << 1, C), at, n, None))
    ws = 1 << 47
    for dw, db in ((at, None), (FREE << 1, at)):
        _refused(L.pulse_keep_wgrad(DESC, T, 64, R(FREE, 64), KEPT, n, dw, db, 0, ws, 1 << 40,
                                    None))
