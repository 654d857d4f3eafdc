"""The conditioned block of the packed-training example: norms, attention,
8-bit checkpoints and 8-bit linear layers together, as a training step and a
sampling step use them, against a float64 block with autograd.

Tolerances (relative L2).  Kept values are off by half a step, uniform; a step is
at most 1 / 63.5 of a group's largest value, which among 32 values is two to three
times their rms: up to 3 / 127 / sqrt(3) = 1.4e-2.  Weight gradients of kept
inputs take that once, fc2's twice (2e-2).  About ten roundings to bf16 on the
way to any result, u / sqrt(3) = 2.3e-3 each with u = 2^-8, add 7e-3.  4e-2 bounds
them all.  8-bit layers: both operands off by half a step of 1 / 127 of the row's
largest, three to four times the rms: 4 / 254 / sqrt(3) = 0.9e-2 each, sqrt(2) of
that a product, and a branch passes two to three products: 3e-2 of the branch."""

import math

import pytest
import torch

from paper_2606_19163_amd import packed_train as pt

from gpu_util import log, rel_l2

pytestmark = pytest.mark.gpu
SHAPES = [(1, 4, 4), (1, 3, 5), (1, 1, 1), (2, 3, 3), (1, 7, 9)]


def _block(lens=None):
    block = pt.ConditionedBlock(SHAPES, heads=4, kv_heads=2, head_dim=48, seed=3)
    block.params["fc1.b"].normal_(0, 0.1)
    block.params["cond.b"].normal_(0, 0.1)
    block.begin(lens)
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*s):
        return torch.randn(*s, generator=g, device="cuda")

    return (block, randn(block.tokens, block.width), randn(len(SHAPES), block.width),
            randn(block.tokens, block.width))


def _reference(block, x, cond):
    """The formulas in float64 with autograd: (out, x, parameters)."""
    p = {n: w.detach().double().cpu().requires_grad_(True) for n, w in block.params.items()}
    x = x.double().cpu().requires_grad_(True)
    mod = cond.double().cpu() @ p["cond"].t() + p["cond.b"]
    dims, at, parts = [block.d - 2 * (block.d // 6 * 2)] + [block.d // 6 * 2] * 2, 0, []
    pos, freq = block.pos.double().cpu(), block.freq.double().cpu()
    for a, n in enumerate(dims):
        parts.append(pos[:, a:a + 1] * freq[at:at + n // 2])
        at += n // 2
    ang = torch.cat(parts, dim=1)[:, None]

    def turn(v):
        a, b = v[..., 0::2], v[..., 1::2]
        c, s = torch.cos(ang), torch.sin(ang)
        return torch.stack([a * c - b * s, a * s + b * c], dim=-1).reshape(v.shape)

    doc = torch.full((block.tokens,), -1)
    off = [0]
    for i, n in enumerate(block.lens):
        doc[off[-1]:off[-1] + n] = i
        off.append(off[-1] + n)
    inside = (doc >= 0).double()[:, None]
    t1, s1, g1, t2, s2, g2 = mod[doc.clamp(min=0)].split(block.width, dim=1)

    def ln(v):
        return torch.nn.functional.layer_norm(v, (block.width,), eps=1e-6)

    u1 = (ln(x) * (1 + s1) + t1) * inside
    qkv = (u1 @ p["qkv"].t()).view(block.tokens, -1, block.d)
    q, k, v = qkv.split([block.h, block.kv, block.kv], dim=1)
    q, k = turn(q), turn(k)
    rep = block.h // block.kv
    o = []
    for i in range(len(block.lens)):
        a, b = off[i], off[i + 1]
        z = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(rep, 1))
        w = torch.softmax(z / math.sqrt(block.d), dim=-1)
        o.append(torch.einsum("hij,jhd->ihd", w, v[a:b].repeat_interleave(rep, 1)))
    o.append(torch.zeros(block.tokens - off[-1], block.h, block.d, dtype=torch.float64))
    y1 = torch.cat(o).reshape(block.tokens, -1) @ p["proj"].t()
    h = x + g1 * y1 * inside
    u2 = (ln(h) * (1 + s2) + t2) * inside
    a = torch.nn.functional.gelu(u2 @ p["fc1"].t() + p["fc1.b"])
    return h + g2 * (a @ p["fc2"].t()) * inside, x, p


@pytest.mark.parametrize("lens", [None, [9, 0, 1, 30, 40]])
def test_block_against_float64(lens):
    block, x, cond, dout = _block(lens)
    out, state = block.forward(x, cond)
    dx = block.backward(dout, state)
    ref, xr, p = _reference(block, x, cond)
    grads = torch.autograd.grad((ref * dout.double().cpu()).sum(), [xr] + list(p.values()))
    assert rel_l2(out.cpu() - x.cpu(), ref.detach() - x.double().cpu()) <= 4e-2
    assert rel_l2(dx.cpu(), grads[0]) <= 4e-2
    for n, g in zip(p, grads[1:]):
        off = rel_l2(block.grads[n].cpu(), g)
        log(f"{n}: {off:.2e}")
        assert off <= 4e-2, (n, off)
    # gradients accumulate
    twice, state = block.forward(x, cond)
    assert torch.equal(twice, out)
    block.backward(dout, state)
    assert rel_l2(block.grads["fc1"].cpu(), 2 * grads[1 + list(p).index("fc1")]) <= 4e-2


def test_block_sampled_with_8_bit_layers():
    block, x, cond, _ = _block([16, 15, 1, 18, 40])
    exact, _, _ = _reference(block, x, cond)
    out = block.sample(x, cond, block.layers8())
    branch = exact.detach() - x.double().cpu()
    assert rel_l2(out.cpu() - x.cpu(), branch) <= 4e-2
    pad = sum(block.lens)
    assert torch.equal(out[pad:], x[pad:])  # padding is left as it was


def test_block_captured_into_a_graph():
    """Forward, backward and sampling replayed with other inputs, next to eager
    calls."""
    block, x, cond, dout = _block()
    layers = block.layers8()

    def work():
        for g in block.grads.values():
            g.zero_()
        out, state = block.forward(x, cond)
        return out, block.backward(dout, state), block.sample(x, cond, layers)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for i in range(3):
        x.mul_(1.1), dout.add_(0.1)
        graph.replay()
        torch.cuda.synchronize()
        grads = {n: g.clone() for n, g in block.grads.items()}
        got_now = [t.clone() for t in got]
        want = work()
        torch.cuda.synchronize()
        for a, b in zip(got_now, want):
            assert torch.equal(a, b), i
        for n, g in block.grads.items():
            # torch's own products and sums run the same kernels on the same inputs
            assert torch.equal(grads[n], g), (i, n)


def test_command_runs():
    first, last, eight = pt.main(["--block", "--steps", "3"])
    assert all(math.isfinite(v) for v in (first, last, eight))
