"""Copies of the operators' objects (copy, deepcopy, pickle): their calls read
their own descriptors and memory, not the original's.  CPU only: tensors are on the
CPU and calls have no rows, so that nothing is launched."""

import copy
import pickle

import pytest
import torch

from paper_2606_19163_amd import ops

from test_ops_host import built  # noqa: F401  (builds the library)

BF = torch.bfloat16


def unpickled(o):
    return pickle.loads(pickle.dumps(o))


@pytest.fixture
def on_cpu(monkeypatch):
    """CPU tensors count as being where the call runs."""
    monkeypatch.setattr(ops, "_here", lambda: (-1, None))


def _none(channels):
    return torch.empty(0, channels, dtype=BF)


@pytest.mark.parametrize("make", [copy.deepcopy, unpickled])
def test_descriptors(make, on_cpu):
    """The original's descriptor is spoilt: a call that read it would refuse."""
    norm, keep = ops.Norm(64), ops.Checkpoint(64, act="gelu")
    n, k = make(norm), make(keep)
    norm.desc.channels = keep.desc.channels = 60
    x = _none(64)
    h, u = n.forward(x, x)
    assert h.shape == u.shape == (0, 64)
    assert k.forward(x)[1].tokens == 0
    del norm, keep
    assert n.forward(x, x)[0].shape == (0, 64) and k.save(x).channels == 64
