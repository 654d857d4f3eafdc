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


# ---- norms: parameters and their gradients ------------------------------------------

X, Y, H, U, DU, DH, DX, DY = ((1 << 32) + (i << 16) for i in range(8))
GATE, SCALE, SHIFT, WEIGHT, BIAS, POST, OFF = ((1 << 33) + (i << 16) for i in range(7))
DGATE, DSCALE, DSHIFT, DWEIGHT, DBIAS, DPOST = ((1 << 34) + (i << 16) for i in range(6))
ROWS = dict(x=X, y=Y, h=H, u=U, du=DU, dh=DH, dx=DX, dy=DY)
PARAMS = dict(offsets=OFF, gate=GATE, scale=SCALE, shift=SHIFT, weight=WEIGHT, bias=BIAS,
              post_weight=POST)
GRADS = dict(dgate=DGATE, dscale=DSCALE, dshift=DSHIFT, dweight=DWEIGHT, dbias=DBIAS,
             dpost_weight=DPOST)
TOKENS, DOCS, CH = 4, 3, 64


def _norm(backward, at):
    """Status of a call whose tensors lie at the addresses above, but for `at`."""
    a = {**ROWS, **PARAMS, **GRADS, **at}
    r = {k: R(a[k], CH) for k in ROWS}
    desc = ops.NormDesc(CH, DOCS, 1, 2, 1, 1e-6, 1.0, S.BF16, S.BF16)
    p = ops.NormParams(gate_stride=CH, scale_stride=CH, shift_stride=CH,
                       **{k: a[k] for k in PARAMS})
    if not backward:
        return ops.lib().pulse_norm_forward(desc, TOKENS, r["x"], r["y"], p, r["h"], r["u"], None)
    return ops.lib().pulse_norm_backward(desc, TOKENS, r["du"], r["dh"], r["h"], r["y"], p,
                                         r["dx"], r["dy"],
                                         ops.NormGrads(**{k: a[k] for k in GRADS}), 1 << 40,
                                         1 << 30, None)


@pytest.mark.parametrize("name", PARAMS)
@pytest.mark.parametrize("backward,out", [(False, "h"), (False, "u"), (True, "dx"), (True, "dy")])
def test_norm_outputs_and_parameters(backward, out, name):
    row = 16 if name == "offsets" else 4 * CH if name.endswith(("weight", "bias")) else 12 * CH
    for at in (ROWS[out], ROWS[out] + TOKENS * CH * 2 - 16, ROWS[out] - row + 16):
        _refused(_norm(backward, {name: at}))


@pytest.mark.parametrize("grad", GRADS)
def test_norm_gradients(grad):
    """The same memory twice, or that of a tensor the call reads or writes."""
    for name, at in {**GRADS, **PARAMS, **{k: ROWS[k] for k in ("du", "dh", "h", "y", "dx",
                                                                 "dy")}}.items():
        if name != grad:
            _refused(_norm(True, {grad: at}))
            if name != "offsets":
                _refused(_norm(True, {grad: at + 4 * CH - 16}))
            _refused(_norm(True, {grad: at - 4 * CH + 16}))
