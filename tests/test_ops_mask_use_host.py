"""Which masks the attention binding takes (no GPU)."""

import pytest
import torch

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import built  # noqa: F401  (builds the library)


def _attn(mask):
    return ops.Attn(mask.queries, 2, 64, keys=mask.keys)._mask(mask, mask.buffer.get_device(), None)


def test_a_mask_that_was_not_built_is_refused():
    m = ops.Mask(70, docs=2, device="cpu")
    with pytest.raises(S.PulseError, match="not built"):
        _attn(m)
    empty = ops.Mask(0, keys=5, docs=1, device="cpu")  # nothing of it is read
    assert _attn(empty) == empty.ptr


@pytest.mark.parametrize("write", [
    lambda m: m.rows.copy_(torch.zeros(70, 4, dtype=torch.int32)),
    lambda m: m.rows[3].fill_(1),
    lambda m: m.rows[:, 1].add_(1),
    lambda m: torch.add(m.rows, 1, out=m.rows),
])
def test_a_mask_written_since_it_was_built_is_refused(write):
    m = ops.Mask(70, docs=2, device="cpu")
    m.stamp = m._stamp()  # as build and from_rows leave it
    assert _attn(m) == m.ptr
    write(m)
    with pytest.raises(S.PulseError, match="from_rows"):
        _attn(m)
    m.stamp = m._stamp()
    assert _attn(m) == m.ptr


def test_a_mask_made_in_inference_mode():
    with torch.inference_mode():
        m = ops.Mask(70, docs=2, device="cpu")
    with pytest.raises(S.PulseError, match="not built"):
        _attn(m)
    m.stamp = m._stamp()
    assert _attn(m) == m.ptr


def _backward(plan, saved, mask):
    t = torch.zeros(plan.qs, dtype=torch.bfloat16)
    plan.backward(t, t, t, t, t, saved, mask)


def test_a_backward_under_a_mask_built_again_is_refused():
    """Refused before any GPU is looked for."""
    m = ops.Mask(70, docs=2, device="cpu")
    plan = ops.Attn(70, 2, 64)
    saved = ops.Saved(2, 70, 64, "cpu")
    with pytest.raises(S.PulseError, match="no forward"):
        _backward(plan, saved, m)
    m._built()
    saved.mask, saved.serial = m, m.serial  # as a forward leaves it
    m._built()
    with pytest.raises(S.PulseError, match="built again"):
        _backward(plan, saved, m)
