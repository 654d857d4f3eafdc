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


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, unpickled])
def test_memory(make, monkeypatch):
    """A copy's addresses are in its own tensors, which hold what the original's do."""
    monkeypatch.setattr(ops.lib(), "pulse_lin8_pack", lambda *a: 0)  # nothing is launched
    monkeypatch.setattr(ops, "_here", lambda: (-1, None))
    kept, saved = ops.Kept(5, 64, "cpu"), ops.Saved(3, 7, 16, "cpu")
    mask = ops.Mask(8, docs=2, device="cpu")
    layer = ops.Linear8(torch.randn(24, 64), bias=torch.randn(24))
    for t in (kept.buffer, layer.weights):
        t.copy_(torch.arange(t.numel()) % 251)
    mask.buffer.copy_(torch.arange(mask.buffer.numel()))
    saved.buffer.copy_(torch.arange(saved.buffer.numel()))
    kept.full, saved.serial, mask.serial = True, 4, 4

    k = make(kept)
    assert k.ptr == k.buffer.data_ptr() != kept.ptr and torch.equal(k.buffer, kept.buffer)
    assert (k.tokens, k.channels, k.bytes, k.home, k.full) == (5, 64, kept.bytes, None, True)

    s = make(saved)
    assert s.lse_ptr == s.buffer.data_ptr() != saved.lse_ptr
    assert s.low_ptr - s.lse_ptr == saved.low_ptr - saved.lse_ptr == 4 * 24
    assert torch.equal(s.lse, saved.lse) and s.serial == 4 and s.mask is None

    m = make(mask)
    assert m.ptr == m.buffer.data_ptr() == m.rows.data_ptr() != mask.ptr
    assert torch.equal(m.rows, mask.rows) and (m.queries, m.keys, m.serial) == (8, 8, 4)

    b = make(layer)
    assert b.ptr == b.weights.data_ptr() != layer.ptr and b.packed == layer.packed
    assert b.bias_ptr == b.bias.data_ptr() != layer.bias_ptr
    assert torch.equal(b.weights, layer.weights) and torch.equal(b.bias, layer.bias)
    b.update(torch.randn(24, 64), None)
    assert b.bias_ptr is None and make(b).bias_ptr is None
    assert layer.bias_ptr == layer.bias.data_ptr()


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, unpickled])
def test_masks_keep_whether_they_were_built(make):
    mask = ops.Mask(8, docs=2, device="cpu")
    with pytest.raises(ops.PulseError, match="not built"):
        make(mask).check()
    mask._built()
    make(mask).check()
    make(make(mask)).check()
    mask.rows.zero_()
    with pytest.raises(ops.PulseError, match="written since"):
        make(mask).check()
    mask._built()
    other = make(mask)
    other.check()
    other.rows.zero_()
    mask.check()
    with pytest.raises(ops.PulseError, match="written since"):
        other.check()


def test_saved_knows_the_mask_it_ran_under():
    mask = ops.Mask(8, docs=2, device="cpu")
    saved = ops.Saved(3, 8, 16, "cpu")
    saved.mask = mask
    assert copy.copy(saved).mask is mask and copy.deepcopy(saved).mask is mask
    m, s, again = copy.deepcopy([mask, saved, saved])
    assert s.mask is m is not mask and again is s
    assert unpickled(saved).mask.queries == 8


def test_masks_of_inference_mode():
    with torch.inference_mode():
        mask = ops.Mask(8, docs=2, device="cpu")
        mask._built()
        copy.deepcopy(mask).check()


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, unpickled])
def test_clips_are_not_copied(make):
    """Two objects would destroy one handle.  Here it is NULL."""
    clip = object.__new__(ops.GradClip)
    clip.h, clip.grads, clip.outs = ops._vp(), [], []
    with pytest.raises(ops.PulseError, match="cannot be copied"):
        make(clip)


class Named(ops.Kept):
    """A subclass with attributes beside the slots."""


@pytest.mark.parametrize("make", [copy.copy, copy.deepcopy, unpickled])
def test_subclasses(make):
    kept = Named(3, 64, "cpu")
    kept.name, kept.full = "u1", True
    k = make(kept)
    assert type(k) is Named and k.name == "u1" and k.full and k.tokens == 3
    assert k.ptr == k.buffer.data_ptr() != kept.ptr
