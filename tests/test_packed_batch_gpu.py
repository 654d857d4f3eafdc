"""Batches of the packed-training example that do not fill their sequence."""

import pytest
import torch

from paper_2606_19163_amd import packed_train
from paper_2606_19163_amd import stage as S

pytestmark = pytest.mark.gpu

SHAPES = [(1, 5, 7), (2, 3, 4), (1, 1, 1)]


def _layer():
    return packed_train.PackedAttention(SHAPES, heads=2, kv_heads=1, head_dim=32)


def test_padding_is_of_no_document():
    layer = _layer()
    layer.begin([20, 0, 11])
    x, target = packed_train.batch(layer, 2)
    assert torch.equal(target[31:], x[31:].float())
    at = 0
    for n in layer.lens:
        d = x[at:at + n].float()
        want = d + d.mean(dim=0) if n else d
        assert torch.allclose(target[at:at + n], want, rtol=1e-5, atol=1e-5)
        at += n
    before = layer.params["qkv"].clone()
    loss, norm = layer.step(x, target, lr=0.1, max_norm=1.0)
    assert torch.isfinite(loss) and torch.isfinite(norm)
    assert not torch.equal(layer.params["qkv"], before)


def test_a_batch_of_the_layers_own_documents_is_as_before():
    layer = _layer()
    layer.begin()
    x, target = packed_train.batch(layer, 5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    y = torch.randn(layer.tokens, 64, generator=gen, device="cuda")
    centre = torch.randn(3, 64, generator=gen, device="cuda")
    doc = torch.tensor([0] * 35 + [1] * 24 + [2], device="cuda")
    assert torch.equal(x, (y + centre[doc]).bfloat16())
    assert target.shape == x.shape


def test_what_does_not_fit_is_refused():
    layer = _layer()
    with pytest.raises(S.PulseError, match="not built"):
        packed_train.batch(layer, 1)
    for lens in ([61, 0, 0], [1, 2], [-1, 2, 3], [1, 2, 3, 4]):
        with pytest.raises(ValueError):
            layer.begin(lens)
