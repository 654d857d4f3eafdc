"""A training step of one attention layer on a packed batch.

    python -m paper_2606_19163_amd.packed_train [--steps N]

Images and clips of several resolutions lie one after another in one sequence.
The layer is a qkv projection, rotary positions over (time, height, width) on
the query and key heads, attention within each document, and an output
projection with a residual.  It learns to add to every token its document's
mean, which only attention can see.  A step is: the mask from the documents'
lengths, forward, backward, the global gradient norm and clipping, and a
plain descent step.  The linear layers are torch's matrix products in bf16
with fp32 masters; everything else runs in the library's kernels.
"""

from __future__ import annotations

import argparse

import torch

from . import ops

#: (time, height, width) of the documents of one batch, in patches
SHAPES = [(1, 16, 16), (1, 12, 20), (1, 32, 32), (4, 9, 16), (1, 1, 1), (2, 13, 7)]


class PackedAttention:
    """h = x + Proj(attention(Rope(x Wqkv))) over documents in one sequence."""

    def __init__(self, shapes, heads, kv_heads, head_dim, cap=30.0, seed=0):
        self.h, self.kv, self.d = heads, kv_heads, head_dim
        self.lens = [t * y * x for t, y, x in shapes]
        self.tokens = sum(self.lens)
        width, rows = heads * head_dim, (heads + 2 * kv_heads) * head_dim
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(out, inp):
            return torch.randn(out, inp, generator=gen, device="cuda") / inp ** 0.5

        self.params = {"qkv": weight(rows, width), "proj": weight(width, width)}
        self.grads = {n: torch.zeros_like(w) for n, w in self.params.items()}
        # a third of each head turns with every axis; pairs of channels, so 2 * n
        third = head_dim // 6 * 2
        dims = [head_dim - 2 * third, third, third]
        self.rope = ops.Rope(heads + kv_heads, head_dim, dims)
        self.freq = ops.rope_freqs(dims)
        self.pos = ops.grid_positions(shapes)
        self.mask = ops.Mask(self.tokens, docs=len(shapes))
        self.attn = ops.Attn(self.tokens, heads, head_dim, kv_heads=kv_heads, cap=cap)
        self.clip = ops.GradClip(self.grads.values())

    def begin(self, lens=None):
        """The batch's mask: every layer of a model would share it.  ``lens``:
        as many documents of other lengths; tokens past them are padding."""
        lens = self.lens if lens is None else list(lens)
        if len(lens) != len(self.lens) or min(lens, default=0) < 0 or sum(lens) > self.tokens:
            raise ValueError(f"{len(self.lens)} documents of {self.tokens} tokens at most, "
                             f"not {lens}")
        self.lens = lens
        off = torch.tensor([0] + lens, device="cuda").cumsum(0).int()
        return self.mask.build(off)

    def forward(self, x):
        """x [tokens, width] bf16; returns h and what the backward needs."""
        w = {n: p.bfloat16() for n, p in self.params.items()}
        qkv = (x @ w["qkv"].t()).view(self.tokens, -1, self.d)
        turned = qkv[:, :self.h + self.kv]
        self.rope.forward(turned, self.pos, self.freq, out=turned)
        q, k, v = qkv.split([self.h, self.kv, self.kv], dim=1)
        o, saved = self.attn.forward(q, k, v, self.mask)
        h = x + o.view(self.tokens, -1) @ w["proj"].t()
        return h, (x, w, qkv, o, saved)

    def backward(self, dh, state):
        """Accumulates the weight gradients; returns dx."""
        x, w, qkv, o, saved = state
        q, k, v = qkv.split([self.h, self.kv, self.kv], dim=1)
        self.grads["proj"] += (dh.t() @ o.view(self.tokens, -1)).float()
        do = (dh @ w["proj"]).view(self.tokens, self.h, self.d)
        dqkv = torch.empty_like(qkv)
        self.attn.backward(do, q, k, v, o, saved, self.mask,
                           out=dqkv.split([self.h, self.kv, self.kv], dim=1))
        turned = dqkv[:, :self.h + self.kv]
        self.rope.backward(turned, self.pos, self.freq, out=turned)
        dqkv = dqkv.view(self.tokens, -1)
        self.grads["qkv"] += (dqkv.t() @ x).float()
        return dh + dqkv @ w["qkv"]

    def step(self, x, target, lr, max_norm):
        """One descent step on the square error, summed over channels and averaged
        over tokens; (its mean over both, gradient norm)."""
        for g in self.grads.values():
            g.zero_()
        h, state = self.forward(x)
        diff = h.float() - target
        loss = (diff * diff).mean()
        self.backward((diff * (2.0 / self.tokens)).bfloat16(), state)
        norm = self.clip.run(max_norm)
        for n, p in self.params.items():
            p.add_(self.grads[n], alpha=-lr)
        return loss, norm


def batch(layer, seed):
    """Tokens and targets: every token plus its document's mean."""
    layer.mask.check()  # layer.begin() was called
    gen = torch.Generator(device="cuda").manual_seed(seed)
    width = layer.h * layer.d
    x = torch.randn(layer.tokens, width, generator=gen, device="cuda")
    centre = torch.randn(len(layer.lens), width, generator=gen, device="cuda")
    doc = layer.mask.rows[:, 3].long()  # the mask knows each row's document
    inside = (doc >= 0)[:, None].float()  # padding has none
    doc = doc.clamp(min=0)
    x = (x + centre[doc] * inside).bfloat16()
    mean = torch.zeros_like(centre).index_add_(0, doc, x.float() * inside)
    mean /= torch.tensor(layer.lens, device="cuda").clamp(min=1)[:, None]
    return x, x.float() + mean[doc] * inside


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)
    layer = PackedAttention(SHAPES, heads=12, kv_heads=4, head_dim=64)
    layer.begin()
    first = last = None
    for i in range(a.steps):
        x, target = batch(layer, i)
        loss, norm = layer.step(x, target, a.lr, a.max_norm)
        if i % 20 == 0 or i == a.steps - 1:
            last = float(loss)
            first = last if first is None else first
            print(f"step {i:4d}  loss {last:.4f}  gradient norm {float(norm):.4f}", flush=True)
    return first, last


if __name__ == "__main__":
    main()
