"""Conditions and weights of documents without rows: whatever they hold, they reach no
gradient, since the sums over rows are empty.  Bit-equal to finite ones."""

import pytest
import torch

from gpu_util import log
from test_norm_gpu import F32, Case

pytestmark = pytest.mark.gpu

#: (rows, offsets, documents without rows): one document, few of many blocks, many
EMPTY = [(0, [0, 0], [0]), (5, [0, 0], [0]), (40, [0, 0, 25, 25, 38], [0, 2]),
         (6000, [0, 2500, 2500, 6000], [1]), (9000, [0, 0, 9000, 9000], [0, 2]),
         (300, [0] * 40 + list(range(0, 240, 2)) + [240] * 9, None)]


@pytest.mark.parametrize("tokens,off,empty", EMPTY)
@pytest.mark.parametrize("channels", [72, 1408])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_conditions_of_documents_without_rows(channels, tokens, off, empty, value):
    log(f"case empty documents {channels} {tokens} {len(off) - 1} {value}")
    if empty is None:
        empty = [d for d in range(len(off) - 1) if off[d] == off[d + 1]]
    c = Case(tokens, channels, off, post="rms", stream=F32)
    h, u = c.forward()
    want = c.backward(h)
    assert all(bool(torch.isfinite(t).all()) for t in want.values())
    for k in ("gate", "scale", "shift"):
        c.dev[k][empty] = value
    h2, u2 = c.forward()
    got = c.backward(h2)
    assert torch.equal(h, h2) and torch.equal(u, u2)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    for k in ("dgate", "dscale", "dshift"):
        assert bool((got[k][empty] == 0).all()), k


@pytest.mark.parametrize("tokens,off", [(0, [0, 0, 0]), (9, [0, 0]), (9, [0, 0, 0])])
def test_weights_without_rows(tokens, off):
    """No document has a row: every gradient of a parameter is 0."""
    c = Case(tokens, 136, off, post="layer")
    for k in ("weight", "bias", "post_weight"):
        c.dev[k].fill_(float("nan"))
    h, _ = c.forward()
    got = c.backward(h)
    for k, v in got.items():
        assert k in ("dx", "dy") or bool((v == 0).all()), k
