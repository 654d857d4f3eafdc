"""Host-side checks of the row operators' C ABI (norms of a block, activations
in 8 bits, 8-bit linear layers; no GPU): every refusal returns its status before
anything is enqueued, and sizes follow the documented layouts.  Pointers here
are addresses that nothing reads."""

import ctypes
import random

import pytest

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import built  # noqa: F401  (builds the library)

P = 1 << 20  # aligned addresses, far enough apart for 4 rows of 64 channels
X, Y, H, U, DU, DH, DX, DY = (P + (i << 16) for i in range(8))
BIG = 1 << 40
R = ops.Rows


def _refused(status, expect):
    assert status == expect, (status, S.lib().pulse_last_error())
    assert S.lib().pulse_last_error()


def _desc(**kw):
    d = dict(channels=64, docs=2, pre=1, post=0, branch=1, eps=1e-6, residual_scale=1.0,
             dtype=S.BF16, stream_dtype=S.BF16)
    return ops.NormDesc(**{**d, **kw})


def _params(**kw):
    d = dict(offsets=P, gate=P, scale=P, shift=P, gate_stride=64, scale_stride=64,
             shift_stride=64)
    return ops.NormParams(**{**d, **kw})


def _fwd(tokens=4, x=None, y=None, h=None, u=None, params=None, desc=None, **kw):
    return ops.lib().pulse_norm_forward(
        desc or _desc(**kw), tokens, x or R(X, 64), y or R(Y, 64), params or _params(),
        h or R(H, 64), u or R(U, 64), None)


def _bwd(tokens=4, ws=BIG, ws_bytes=1 << 30, grads=None, params=None, desc=None, rows=None, **kw):
    r = dict(du=R(DU, 64), dh=R(DH, 64), h=R(H, 64), y=R(Y, 64), dx=R(DX, 64), dy=R(DY, 64))
    r.update(rows or {})
    return ops.lib().pulse_norm_backward(
        desc or _desc(**kw), tokens, r["du"], r["dh"], r["h"], r["y"], params or _params(),
        r["dx"], r["dy"], grads or ops.NormGrads(P, P, P, None, None, None), ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(channels=0), dict(channels=60), dict(channels=8200),
                                dict(docs=0), dict(docs=(1 << 20) + 1), dict(tokens=-1),
                                dict(tokens=(1 << 23) + 1)])
def test_norm_shapes(kw):
    _refused(_fwd(**kw), S.E_SHAPE)
    _refused(_bwd(**kw), S.E_SHAPE)


@pytest.mark.parametrize("kw", [
    dict(pre=3), dict(post=-1), dict(branch=2), dict(branch=0, post=1), dict(branch=0, pre=0),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(residual_scale=float("nan")), dict(residual_scale=float("inf")), dict(dtype=2),
    dict(stream_dtype=5), dict(dtype=S.F32, stream_dtype=S.BF16),
    dict(params=_params(offsets=None)), dict(params=_params(offsets=P + 2)),
    dict(params=_params(gate=P + 4)), dict(params=_params(scale_stride=66)),
    dict(params=_params(shift_stride=-64)), dict(params=_params(gate_stride=(1 << 40) + 4)),
    dict(params=_params(weight=P + 8)), dict(params=_params(post_weight=P)),
    dict(pre=0, params=_params(shift=None)), dict(pre=0, params=_params(scale=None)),
    dict(branch=0),
])
def test_norm_arguments(kw):
    _refused(_fwd(**kw), S.E_INVALID_ARG)
    _refused(_bwd(**kw), S.E_INVALID_ARG)


@pytest.mark.parametrize("kw", [
    dict(x=R(None, 64)), dict(x=R(X + 8, 64)), dict(y=R(Y, 60)), dict(h=R(H, -64)),
    dict(u=R(U, 32)), dict(h=R(H, 0)), dict(u=R(U, 1 << 41)), dict(h=R(X + 16, 64)),
    dict(u=R(X, 64)), dict(u=R(H, 64)), dict(h=R(Y, 64)), dict(u=R(Y, 128)),
    dict(h=R(X, 128), x=R(X, 64)), dict(u=R(H + 64, 128), h=R(H, 128)),
])
def test_norm_forward_tensors(kw):
    _refused(_fwd(**kw), S.E_INVALID_ARG)


def test_norm_null_structures():
    L = ops.lib()
    r = R(X, 64)
    for args in ((None, 4, r, r, _params(), r, r, None), (_desc(), 4, None, r, _params(), r, r, None),
                 (_desc(), 4, r, None, _params(), r, r, None), (_desc(), 4, r, r, None, r, r, None),
                 (_desc(), 4, r, R(Y, 64), _params(), None, r, None),
                 (_desc(), 4, r, R(Y, 64), _params(), R(H, 64), None, None)):
        _refused(L.pulse_norm_forward(*args), S.E_INVALID_ARG)
    n = ctypes.c_size_t()
    _refused(L.pulse_norm_sizes(None, 4, n), S.E_INVALID_ARG)
    _refused(L.pulse_norm_sizes(_desc(), 4, None), S.E_INVALID_ARG)
    _refused(L.pulse_norm_sizes(_desc(), -1, n), S.E_SHAPE)


@pytest.mark.parametrize("kw", [
    dict(ws=None), dict(ws=BIG + 16), dict(ws_bytes=64),
    dict(rows=dict(du=None)), dict(rows=dict(h=None)), dict(rows=dict(y=None)),
    dict(rows=dict(dy=None)), dict(rows=dict(dx=R(DX, 32))), dict(rows=dict(dx=R(DU, 64))),
    dict(rows=dict(dx=R(H, 64))), dict(rows=dict(dy=R(DH, 64))), dict(rows=dict(dy=R(DX, 64))),
    dict(rows=dict(dy=R(H, 64))), dict(rows=dict(dx=R(Y, 64))), dict(rows=dict(dh=R(DH + 2, 64))),
    dict(grads=ops.NormGrads(P + 4, P, P, None, None, None)),
    dict(grads=ops.NormGrads(P, P, P, None, None, P)),
    dict(pre=0, params=_params(scale=None, shift=None)),
])
def test_norm_backward_tensors(kw):
    _refused(_bwd(**kw), S.E_INVALID_ARG)


def test_norm_sizes_hold_the_sums():
    """Three fp32 rows for every block and document, at least."""
    n = ctypes.c_size_t()
    for c, docs, tokens in ((64, 1, 0), (64, 1, 1), (1408, 8, 8192), (8192, 1000, 5),
                            (320, 1 << 20, 1 << 23)):
        assert ops.lib().pulse_norm_sizes(_desc(channels=c, docs=docs), tokens, n) == S.OK
        assert n.value >= 12 * c * docs * 2
        assert n.value <= 12 * c * (docs * 2 + 520 + (tokens + 3) // 4) + 4096


# ---- kept rows --------------------------------------------------------------------


def _keep_size(channels, tokens):
    n = ctypes.c_size_t()
    return ops.lib().pulse_keep_sizes(ops.KeepDesc(channels, 0, S.BF16), tokens, n), n.value


def test_keep_sizes():
    for c, t in ((8, 1), (32, 3), (40, 7), (1408, 8192), (65536, 1 << 23), (64, 0)):
        p = -(-c // 32) * 32
        assert _keep_size(c, t) == (S.OK, -(-t * p // 16) * 16 + t * -(-p // 128) * 4)
    for c, t in ((0, 1), (12, 1), (65544, 1), (64, -1), (64, (1 << 23) + 1)):
        _refused(_keep_size(c, t)[0], S.E_SHAPE)
    _refused(ops.lib().pulse_keep_sizes(None, 1, ctypes.c_size_t()), S.E_INVALID_ARG)
    _refused(ops.lib().pulse_keep_sizes(ops.KeepDesc(64, 0, 0), 1, None), S.E_INVALID_ARG)


K, K2 = BIG, BIG + (1 << 20)


@pytest.mark.parametrize("kw", [
    dict(act=3), dict(act=-1), dict(dtype=2), dict(kept=None), dict(kept=K + 8),
    dict(kept_bytes=100), dict(x=R(None, 64)), dict(x=R(X + 2, 64)), dict(x=R(X, 60)),
    dict(a=R(Y, 32)), dict(a=R(X + 16, 64)), dict(a=R(X, 128)), dict(act=0), dict(kept=X),
    dict(a=R(K, 64)),
])
def test_keep_save(kw):
    d = dict(x=R(X, 64), a=R(Y, 64), kept=K, kept_bytes=1 << 12, act=1, dtype=S.BF16)
    d.update(kw)
    L = ops.lib()
    _refused(L.pulse_keep_save(ops.KeepDesc(64, d["act"], d["dtype"]), 4, d["x"], d["a"],
                               d["kept"], d["kept_bytes"], None), S.E_INVALID_ARG)


@pytest.mark.parametrize("kw", [
    dict(act=0), dict(da=R(None, 64)), dict(dx=R(DX, 0)), dict(dx=R(DU + 16, 64)),
    dict(kept=None), dict(kept_bytes=0), dict(again=K), dict(again=K2 + 4), dict(dx=R(K, 64)),
    dict(again=DU), dict(again=DX), dict(again_bytes=8),
])
def test_keep_backward(kw):
    d = dict(da=R(DU, 64), dx=R(DX, 64), kept=K, kept_bytes=1 << 12, again=K2,
             again_bytes=1 << 12, act=2)
    d.update(kw)
    _refused(ops.lib().pulse_keep_backward(
        ops.KeepDesc(64, d["act"], S.BF16), 4, d["da"], d["kept"], d["kept_bytes"], d["dx"],
        d["again"], d["again_bytes"], None), S.E_INVALID_ARG)


def test_keep_load():
    L, desc = ops.lib(), ops.KeepDesc(64, 0, S.BF16)
    for kept, n, x in ((None, 4096, R(X, 64)), (K, 12, R(X, 64)), (K, 4096, R(X, 32)),
                       (K, 4096, R(K, 64)), (K, 4096, None)):
        _refused(L.pulse_keep_load(desc, 4, kept, n, x, None), S.E_INVALID_ARG)
    _refused(L.pulse_keep_load(desc, -1, K, 4096, R(X, 64), None), S.E_SHAPE)


def _wgrad(outputs=48, tokens=4, dy=None, kept=K, dw=X, db=Y, accumulate=0, ws=BIG << 1,
           ws_bytes=1 << 30):
    return ops.lib().pulse_keep_wgrad(ops.KeepDesc(64, 0, S.BF16), tokens, outputs,
                                      dy or R(DU, 64), kept, 1 << 12, dw, db, accumulate, ws,
                                      ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(dy=R(None, 64)), dict(dy=R(DU, 60)), dict(dy=R(DU + 8, 64)), dict(kept=None),
    dict(dw=None), dict(dw=X + 8), dict(db=Y + 4), dict(accumulate=2), dict(ws=None),
    dict(ws=(BIG << 1) + 16), dict(ws_bytes=16), dict(dw=DU), dict(db=DU), dict(dw=K), dict(db=K),
    dict(db=X),
])
def test_weight_grad(kw):
    _refused(_wgrad(**kw), S.E_INVALID_ARG)


def test_weight_grad_shapes():
    for kw in (dict(outputs=0), dict(outputs=12), dict(outputs=65544), dict(tokens=-1),
               dict(tokens=(1 << 23) + 1)):
        _refused(_wgrad(**kw), S.E_SHAPE)
    n = ctypes.c_size_t()
    d = ops.KeepDesc(64, 0, S.BF16)
    _refused(ops.lib().pulse_keep_wgrad_sizes(d, 4, 12, n), S.E_SHAPE)
    _refused(ops.lib().pulse_keep_wgrad_sizes(d, 4, 16, None), S.E_INVALID_ARG)


def test_weight_grad_workspace_over_shapes():
    """The workspace stays bounded whatever the sizes.  There are splits only
    while their tiles do not fill the GPU: fp32 partial gradients of at most 512
    tiles of 128 x 128, 32 MB, and the columns' sums beside them (65536 outputs of 512
    splits or channel tiles: 128 MB).  Fragments of x take at most 512 MB, since
    more tokens are taken in parts."""
    rng = random.Random(3)
    n = ctypes.c_size_t()
    for _ in range(3000):
        c, m = (8 * int(2 ** rng.uniform(0, 13)) for _ in range(2))
        t = int(2 ** rng.uniform(0, 23))
        assert ops.lib().pulse_keep_wgrad_sizes(ops.KeepDesc(c, 0, S.BF16), t, m, n) == S.OK
        assert n.value <= 700 << 20, (c, m, t, n.value)


# ---- 8-bit linear layers -------------------------------------------------------------


def _lin8_sizes(inputs=64, outputs=48, act=0, dtype=S.BF16, tokens=4):
    w, b = ctypes.c_size_t(), ctypes.c_size_t()
    return ops.lib().pulse_lin8_sizes(ops.Lin8Desc(inputs, outputs, act, dtype), tokens, w,
                                      b), w.value, b.value


@pytest.mark.parametrize("kw", [dict(inputs=0), dict(inputs=12), dict(inputs=65544),
                                dict(outputs=4), dict(outputs=65544), dict(tokens=-1),
                                dict(tokens=(1 << 23) + 1),
                                dict(tokens=1 << 23, outputs=65536)])
def test_lin8_shapes(kw):
    _refused(_lin8_sizes(**kw)[0], S.E_SHAPE)


def test_lin8_sizes():
    for kw in (dict(act=3), dict(dtype=S.F32)):
        _refused(_lin8_sizes(**kw)[0], S.E_INVALID_ARG)
    _refused(ops.lib().pulse_lin8_sizes(None, 1, None, None), S.E_INVALID_ARG)
    st, w, b = _lin8_sizes(1408, 8448, tokens=1)
    assert st == S.OK and w >= 1408 * 8448 + 4 * 8448
    assert b == 0  # few tokens are laid out by every block for itself
    assert _lin8_sizes(1408, 8448, tokens=40)[2] >= 40 * (1408 + 4)
    assert _lin8_sizes(tokens=0)[2] == 0


W = BIG << 2


def _lin8(tokens=40, x=None, y=None, weights=W, weight_bytes=1 << 20, bias=P, ws=BIG << 1,
          ws_bytes=1 << 20):
    return ops.lib().pulse_lin8_forward(ops.Lin8Desc(64, 48, 0, S.BF16), tokens, x or R(X, 64),
                                        weights, weight_bytes, bias, y or R(Y, 48), ws, ws_bytes,
                                        None)


@pytest.mark.parametrize("kw", [
    dict(x=R(None, 64)), dict(x=R(X + 8, 64)), dict(x=R(X, 63)), dict(y=R(Y, 40)),
    dict(y=R(X, 64)), dict(y=R(X + 1024, 64)), dict(weights=None), dict(weights=W + 16),
    dict(weight_bytes=64), dict(bias=P + 4), dict(ws=None), dict(ws=(BIG << 1) + 4),
    dict(ws_bytes=64),
])
def test_lin8_forward(kw):
    _refused(_lin8(**kw), S.E_INVALID_ARG)


def test_lin8_pack():
    d = ops.Lin8Desc(64, 48, 0, S.BF16)
    for w, dt, to, n in ((None, 0, W, 1 << 20), (P + 2, 0, W, 1 << 20), (P, 3, W, 1 << 20),
                         (P, 0, None, 1 << 20), (P, 0, W + 8, 1 << 20), (P, 0, W, 100)):
        _refused(ops.lib().pulse_lin8_pack(d, w, dt, to, n, None), S.E_INVALID_ARG)
    _refused(ops.lib().pulse_lin8_pack(None, P, 0, W, 1 << 20, None), S.E_INVALID_ARG)


# ---- the binding ------------------------------------------------------------------


@pytest.mark.parametrize("make", [
    lambda: ops.Norm(60), lambda: ops.Norm(64, pre="batch"), lambda: ops.Norm(64, post="none"),
    lambda: ops.Norm(64, branch=False, pre=None), lambda: ops.Norm(64, docs=0),
    lambda: ops.Checkpoint(12), lambda: ops.Checkpoint(64, act="relu"),
])
def test_binding_refuses(make):
    with pytest.raises(S.PulseError):
        make()


def test_no_tokens_need_no_memory():
    """Calls of no rows check their descriptors only."""
    L, none = ops.lib(), R(None, 0)
    assert L.pulse_norm_forward(_desc(), 0, none, none, _params(), none, none, None) == S.OK
    d = ops.KeepDesc(64, 1, S.BF16)
    assert L.pulse_keep_save(d, 0, none, none, None, 0, None) == S.OK
    assert L.pulse_keep_load(d, 0, None, 0, none, None) == S.OK
    assert L.pulse_keep_backward(d, 0, none, None, 0, none, None, 0, None) == S.OK
    assert L.pulse_lin8_forward(ops.Lin8Desc(64, 48, 0, S.BF16), 0, none, W, 1 << 20, None, none,
                                None, 0, None) == S.OK
