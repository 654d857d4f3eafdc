"""Tensors with another number of axes are refused as the other arguments are.  CPU
only: nothing is launched."""

import pytest
import torch

from paper_2606_19163_amd import ops

from test_ops_host import built  # noqa: F401  (builds the library)

BF = torch.bfloat16


@pytest.mark.parametrize("shape", [(0,), (0, 2, 8)])
def test_axes(shape, monkeypatch):
    monkeypatch.setattr(ops, "_here", lambda: (-1, None))
    bad, none = torch.empty(shape, dtype=BF), torch.empty(0, 64, dtype=BF)
    keep, norm = ops.Checkpoint(64, act="gelu"), ops.Norm(64)
    kept = ops.Kept(0, 64, "cpu")
    kept.full = True
    for fn in (lambda: keep.weight_grad(bad, kept), lambda: keep.save(bad, kept=kept),
               lambda: keep.forward(bad), lambda: keep.backward(bad, kept),
               lambda: norm.forward(bad, none), lambda: norm.forward(none, bad),
               lambda: norm.backward(bad, none, y=none), lambda: norm.backward(none, bad, y=none)):
        with pytest.raises(ops.PulseError):
            fn()
