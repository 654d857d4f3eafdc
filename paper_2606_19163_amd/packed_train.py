"""A training step of one attention layer on a packed batch, or of a whole
conditioned block.

    python -m paper_2606_19163_amd.packed_train [--steps N] [--block]

Images and clips of several resolutions lie one after another in one sequence.
The layer is a qkv projection, rotary positions over (time, height, width) on
the query and key heads, attention within each document, and an output
projection with a residual.  It learns to add to every token its document's
mean, which only attention can see.  A step is: the mask from the documents'
lengths, forward, backward, the global gradient norm and clipping, and a
plain descent step.  The linear layers are torch's matrix products in bf16
with fp32 masters; everything else runs in the library's kernels.

With ``--block`` the layer is a transformer block whose norms are scaled,
shifted and gated by each document's condition, and what its backward pass needs
of the linear layers' inputs is kept in 8 bits; at the end its output is
sampled with 8-bit linear layers.
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


class ConditionedBlock(PackedAttention):
    """A transformer block on documents with a condition each:

        u1 = LN(x) (1 + s1) + t1      y1 = Proj(attention(Rope(u1 Wqkv)))
        h  = x + g1 y1                u2 = LN(h) (1 + s2) + t2
        y2 = Fc2(GELU(Fc1(u2)))       out = h + g2 y2

    where (t1, s1, g1, t2, s2, g2) of a document are a linear layer of its
    condition.  The stream x is fp32.  The inputs of qkv, fc1 and fc2 are kept in 8
    bits between the passes (that of fc2 is computed again from fc1's output)."""

    def __init__(self, shapes, heads, kv_heads, head_dim, mlp_ratio=4, cap=0.0, seed=0):
        super().__init__(shapes, heads, kv_heads, head_dim, cap, seed)
        width, docs = heads * head_dim, len(shapes)
        self.width, self.hidden = width, mlp_ratio * width
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)

        def weight(out, inp):
            return torch.randn(out, inp, generator=gen, device="cuda") / inp ** 0.5

        self.params["fc1"] = weight(self.hidden, width)
        self.params["fc1.b"] = torch.zeros(self.hidden, device="cuda")
        self.params["fc2"] = weight(width, self.hidden)
        self.params["cond"] = 0.3 * weight(6 * width, width)
        self.params["cond.b"] = torch.zeros(6 * width, device="cuda")
        self.grads = {n: torch.zeros_like(w) for n, w in self.params.items()}
        self.clip = ops.GradClip(self.grads.values())
        f32 = torch.float32
        self.norms = [ops.Norm(width, docs=docs, branch=False, stream_dtype=f32),
                      ops.Norm(width, docs=docs, stream_dtype=f32),
                      ops.Norm(width, docs=docs, pre=None, stream_dtype=f32)]
        self.keep, self.gelu = ops.Checkpoint(width), ops.Checkpoint(self.hidden, act="gelu")

    def begin(self, lens=None):
        rows = super().begin(lens)
        self.offsets = torch.tensor([0] + self.lens, device="cuda").cumsum(0).int()
        return rows

    def _attend(self, qkv, keep):
        """Attention of a projection's output, turned in place."""
        qkv = qkv.view(self.tokens, -1, self.d)
        turned = qkv[:, :self.h + self.kv]
        self.rope.forward(turned, self.pos, self.freq, out=turned)
        q, k, v = qkv.split([self.h, self.kv, self.kv], dim=1)
        o, saved = self.attn.forward(q, k, v, self.mask, keep=keep)
        return o.view(self.tokens, -1), saved, qkv

    def _halves(self, x, mod, attend, mlp):
        """out and the streams and inputs between, with the two halves given."""
        t1, s1, g1, t2, s2, g2 = mod.split(self.width, dim=1)
        n0, n1, n2 = self.norms
        _, u1 = n0.forward(x, offsets=self.offsets, scale=s1, shift=t1)
        y1 = attend(u1)
        h, u2 = n1.forward(x, y1, offsets=self.offsets, gate=g1, scale=s2, shift=t2)
        y2 = mlp(u2)
        out, _ = n2.forward(h, y2, offsets=self.offsets, gate=g2)
        return out, (x, u1, y1, h, u2, y2)

    def forward(self, x, cond):
        """x [tokens, width] fp32 and cond [docs, width] fp32; returns out and
        what the backward needs."""
        w = {n: p.bfloat16() for n, p in self.params.items()}
        mod = cond @ self.params["cond"].t() + self.params["cond.b"]
        kept, mid = {}, {}

        def attend(u1):
            kept["u1"] = self.keep.save(u1)
            mid["o"], mid["saved"], mid["qkv"] = self._attend(u1 @ w["qkv"].t(), True)
            return mid["o"] @ w["proj"].t()

        def mlp(u2):
            kept["u2"] = self.keep.save(u2)
            a, kept["z"] = self.gelu.forward(torch.addmm(w["fc1.b"], u2, w["fc1"].t()))
            return a @ w["fc2"].t()

        out, (_, _, y1, h, _, y2) = self._halves(x, mod, attend, mlp)
        return out, (x, cond, w, mod, y1, h, y2, kept, mid)

    def backward(self, dout, state):
        """Accumulates the weight gradients; returns dx."""
        x, cond, w, mod, y1, h, y2, kept, mid = state
        t1, s1, g1, t2, s2, g2 = mod.split(self.width, dim=1)
        n0, n1, n2 = self.norms
        off = self.offsets
        r2 = n2.backward(None, None, dh=dout, y=y2, offsets=off, gate=g2)
        again = self.gelu.buffer(self.tokens)
        dz = self.gelu.backward(r2["dy"] @ w["fc2"], kept["z"], again=again)
        self.gelu.weight_grad(r2["dy"], again, out=self.grads["fc2"], accumulate=True)
        self.keep.weight_grad(dz, kept["u2"], out=self.grads["fc1"],
                              bias_out=self.grads["fc1.b"], accumulate=True)
        r1 = n1.backward(dz @ w["fc1"], h, dh=r2["dx"], y=y1, offsets=off, gate=g1, scale=s2,
                         shift=t2)
        self.grads["proj"] += (r1["dy"].t() @ mid["o"]).float()
        heads = (self.tokens, self.h, self.d)
        qkv, dqkv = mid["qkv"], torch.empty_like(mid["qkv"])
        split = [self.h, self.kv, self.kv]
        self.attn.backward((r1["dy"] @ w["proj"]).view(heads), *qkv.split(split, dim=1),
                           mid["o"].view(heads), mid["saved"], self.mask,
                           out=dqkv.split(split, dim=1))
        turned = dqkv[:, :self.h + self.kv]
        self.rope.backward(turned, self.pos, self.freq, out=turned)
        dqkv = dqkv.view(self.tokens, -1)
        self.keep.weight_grad(dqkv, kept["u1"], out=self.grads["qkv"], accumulate=True)
        r0 = n0.backward(dqkv @ w["qkv"], x, dh=r1["dx"], offsets=off, scale=s1, shift=t1)
        dmod = torch.cat([r0["dshift"], r0["dscale"], r1["dgate"], r1["dshift"], r1["dscale"],
                          r2["dgate"]], dim=1)
        self.grads["cond"] += dmod.t() @ cond
        self.grads["cond.b"] += dmod.sum(dim=0)
        return r0["dx"]

    def step(self, x, target, cond, lr, max_norm):
        """One descent step on the square error, as the attention layer's."""
        for g in self.grads.values():
            g.zero_()
        out, state = self.forward(x, cond)
        diff = out - target
        loss = (diff * diff).mean()
        self.backward(diff * (2.0 / self.tokens), state)
        norm = self.clip.run(max_norm)
        for n, p in self.params.items():
            p.add_(self.grads[n], alpha=-lr)
        return loss, norm

    def layers8(self):
        """The linear layers in 8-bit integers, of the weights as they are."""
        p = self.params
        return {"qkv": ops.Linear8(p["qkv"]), "proj": ops.Linear8(p["proj"]),
                "fc1": ops.Linear8(p["fc1"], bias=p["fc1.b"], act="gelu"),
                "fc2": ops.Linear8(p["fc2"]), "cond": ops.Linear8(p["cond"], bias=p["cond.b"])}

    def sample(self, x, cond, layers):
        """out with the layers of :meth:`layers8`, and nothing kept."""
        mod = layers["cond"].forward(cond.bfloat16()).float()

        def attend(u1):
            return layers["proj"].forward(self._attend(layers["qkv"].forward(u1), False)[0])

        def mlp(u2):
            return layers["fc2"].forward(layers["fc1"].forward(u2))

        return self._halves(x, mod, attend, mlp)[0]


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


def train_block(steps, lr, max_norm):
    """Trains the block on the same task, where a document's mean is also its
    condition, and samples it with 8-bit layers; (first loss, last loss, that of
    the 8-bit output)."""
    block = ConditionedBlock(SHAPES, heads=12, kv_heads=4, head_dim=64)
    block.begin()
    first = last = None
    for i in range(steps):
        x, target = batch(block, i)
        cond = torch.nn.functional.normalize(target - x.float(), dim=1)[block.offsets[:-1].long()]
        loss, norm = block.step(x.float(), target, cond * block.width ** 0.5, lr, max_norm)
        if i % 20 == 0 or i == steps - 1:
            last = float(loss)
            first = last if first is None else first
            print(f"step {i:4d}  loss {last:.4f}  gradient norm {float(norm):.4f}", flush=True)
    out = block.sample(x.float(), cond * block.width ** 0.5, block.layers8())
    eight = float(((out - target) ** 2).mean())
    print(f"8-bit linear layers after the last step: loss {eight:.4f}", flush=True)
    return first, last, eight


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--block", action="store_true", help="a whole conditioned block")
    a = ap.parse_args(argv)
    if a.block:
        return train_block(a.steps, 0.2 * a.lr, a.max_norm)
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
