"""The packed-batch training example: its gradients against torch's autograd
of the same layer in float64, and a loss that falls."""

import math

import pytest
import torch

from paper_2606_19163_amd import ops, packed_train

from gpu_util import log, rel_l2

pytestmark = pytest.mark.gpu


def _reference(layer, x, target):
    """Loss and weight gradients of the layer in float64 (weights and tokens
    as the layer's matrix products see them), document by document."""
    w = {n: p.bfloat16().double().cpu().requires_grad_() for n, p in layer.params.items()}
    x, target = x.double().cpu(), target.double().cpu()
    h, kv, d = layer.h, layer.kv, layer.d
    dims = list(layer.rope.desc.axis_dim)[:3]
    axis = sum([[a] * (n // 2) for a, n in enumerate(dims)], [])
    ang = layer.pos.double().cpu()[:, axis] * layer.freq.double().cpu()
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    qkv = (x @ w["qkv"].t()).view(len(x), -1, d)
    t = qkv[:, :h + kv]
    a, b = t[..., 0::2], t[..., 1::2]
    t = torch.stack([a * c - b * s, a * s + b * c], dim=-1).reshape(t.shape)
    q, k, v = t[:, :h], t[:, h:], qkv[:, h + kv:]
    out, at = [], 0
    for n in layer.lens:
        r = slice(at, at + n)
        heads = []
        for i in range(h):
            z = q[r, i] @ k[r, i // (h // kv)].t() / math.sqrt(d)
            p = torch.softmax(30.0 * torch.tanh(z / 30.0), dim=-1)
            heads.append(p @ v[r, i // (h // kv)])
        out.append(torch.stack(heads, dim=1))
        at += n
    y = x + torch.cat(out).reshape(len(x), -1) @ w["proj"].t()
    loss = ((y - target) ** 2).sum() / len(x)
    loss.backward()
    return float(((y - target) ** 2).mean().detach()), {n: p.grad for n, p in w.items()}


def test_gradients_of_the_layer():
    shapes = [(1, 5, 7), (2, 3, 4), (1, 1, 1), (1, 9, 9)]
    layer = packed_train.PackedAttention(shapes, heads=4, kv_heads=2, head_dim=32)
    rows = layer.begin().cpu()
    assert rows[:, 3].tolist() == sum([[i] * n for i, n in enumerate(layer.lens)], [])
    x, target = packed_train.batch(layer, 3)
    before = {n: p.clone() for n, p in layer.params.items()}
    loss, grads = _reference(layer, x, target)
    got, norm = layer.step(x, target, lr=0.125, max_norm=1e9)
    assert abs(float(got) - loss) <= 1e-2 * loss
    # bf16 activations, gradients and products: each of about ten tensors in
    # the chain is rounded once, 2.3e-3 each in the relative L2 norm
    for n, g in grads.items():
        e = rel_l2(layer.grads[n].cpu(), g)
        log(f"  {n}: {e:.2e}")
        assert e <= 3e-2, n
    n2 = math.sqrt(sum(float((g.double() ** 2).sum()) for g in layer.grads.values()))
    assert abs(float(norm) - n2) <= 1e-6 * n2
    for n, p in layer.params.items():
        assert torch.allclose(p, before[n] - 0.125 * layer.grads[n], rtol=1e-6, atol=1e-7)


def test_clipping_bounds_the_step():
    layer = packed_train.PackedAttention([(1, 4, 4)], heads=2, kv_heads=1, head_dim=32)
    layer.begin()
    x, target = packed_train.batch(layer, 1)
    _, norm = layer.step(x, target, lr=0.0, max_norm=1e-3)
    assert float(norm) > 1e-3
    assert abs(float(ops.GradClip(layer.grads.values()).run(1.0)) - 1e-3) <= 1e-8


def test_training_lowers_the_loss():
    first, last = packed_train.main(["--steps", "61"])
    assert last < 0.8 * first
