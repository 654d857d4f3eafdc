"""Norms of a block with gate and residual against a float64 form of the same
formulas, forward and backward.

Tolerances.  A result is computed in fp32 and rounded once: off by half a step
(2^-8 of the value in bf16, 2^-24 in fp32), and by fp32's roundings before.
Those are sums over C channels (a row's statistics; at most C / 64 + 6 roundings
in a row, so below 2^-24 * 140 = 8e-6 of the sum of absolute terms) and over
rows (at most rows / 4 + 40 in a row; 2e-5 for the 1200 of the longest case,
a hundredth of that where roundings have either sign).  SLACK = 1e-5 times the
largest value of the tensor covers both.  h in bf16 is compared with half a
step; u and the gradients are those of h as the kernel rounded it, so they are
computed from the kernel's own h."""

import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SLACK = 1e-5


def _close(got, ref, what):
    got, ref = got.detach().cpu(), ref.detach()
    assert got.shape == ref.shape, what
    step = 2.0 ** -8 if got.dtype == BF else 2.0 ** -24
    bound = step * ref.abs() + SLACK * ref.abs().max() + 1e-30
    off = (got.double() - ref).abs()
    assert bool((off <= bound).all()), (what, float((off / bound).max()))


def _norm(v, kind, w, b, eps):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    n = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    n = n if w is None else n * w
    return n if b is None else n + b


def _docs(off, tokens):
    """Document of every row, -1 for none."""
    d = torch.full((tokens,), -1)
    for i in range(len(off) - 1):
        d[off[i]:off[i + 1]] = i
    return d


class Case:
    def __init__(self, tokens, channels, off=None, pre="layer", post=None, branch=True,
                 conds="gsf", affine=True, dtype=BF, stream=F32, eps=1e-6, r=0.7, seed=0):
        g = torch.Generator().manual_seed(seed + tokens + channels)

        def randn(*s):
            return torch.randn(s, generator=g, dtype=F32)

        self.t, self.c, self.off, self.pre, self.post = tokens, channels, off, pre, post
        self.eps, self.r = eps, r
        docs = 1 if off is None else len(off) - 1
        self.doc = torch.zeros(tokens, dtype=torch.long) if off is None else _docs(off, tokens)
        wide = torch.exp(0.5 * randn(channels))
        self.x = ((randn(tokens, channels) + 0.3) * wide).to(stream)
        self.y = randn(tokens, channels).to(dtype) if branch else None
        self.du = randn(tokens, channels).to(dtype) if pre else None
        self.dh = randn(tokens, channels).to(stream)
        self.p = dict(gate=0.5 * randn(docs, channels) if "g" in conds and branch else None,
                      scale=0.5 * randn(docs, channels) if "s" in conds and pre else None,
                      shift=randn(docs, channels) if "f" in conds and pre else None,
                      weight=1 + 0.2 * randn(channels) if affine and pre else None,
                      bias=0.2 * randn(channels) if affine and pre else None,
                      post_weight=1 + 0.2 * randn(channels) if affine and post else None)
        self.plan = ops.Norm(channels, docs=docs, pre=pre, post=post, branch=branch, eps=eps,
                             residual_scale=r, dtype=dtype, stream_dtype=stream)
        self.dev = {k: None if v is None else v.cuda() for k, v in self.p.items()}
        if off is not None:
            self.dev["offsets"] = torch.tensor(off, dtype=torch.int32, device="cuda")

    def cuda(self, name):
        v = getattr(self, name)
        return None if v is None else v.cuda()

    def forward(self, **kw):
        return self.plan.forward(self.cuda("x"), self.cuda("y"), **self.dev, **kw)

    def backward(self, h, **kw):
        return self.plan.backward(self.cuda("du"), None if self.pre is None else h,
                                  dh=self.cuda("dh"), y=self.cuda("y"), **self.dev, **kw)

    def reference(self, h):
        """(h of the formula, u of `h`, gradients at `h`)."""
        inside = self.doc >= 0
        doc = self.doc.clamp(min=0)
        par = {k: None if v is None else v.double().requires_grad_(True)
               for k, v in self.p.items()}
        y = None if self.y is None else self.y.double().requires_grad_(True)
        step = torch.zeros(self.t, self.c, dtype=torch.float64)
        if y is not None:
            py = y if self.post is None else _norm(y, self.post, par["post_weight"], None, self.eps)
            gate = self.r if par["gate"] is None else self.r * par["gate"][doc]
            step = torch.where(inside[:, None], gate * py, torch.zeros_like(py))
        h_ref = self.x.double() + step.detach()
        base = (h.double().cpu() - step.detach()).requires_grad_(True)
        hh = base + step
        loss = (hh * self.dh.double()).sum()
        u = None
        if self.pre:
            u = _norm(hh, self.pre, par["weight"], par["bias"], self.eps)
            if par["scale"] is not None:
                u = u * (1 + par["scale"][doc])
            if par["shift"] is not None:
                u = u + par["shift"][doc]
            u = torch.where(inside[:, None], u, torch.zeros_like(u))
            loss = loss + (u * self.du.double()).sum()
        leaves = {"dx": base}
        if y is not None:
            leaves["dy"] = y
        leaves.update({"d" + k: v for k, v in par.items() if v is not None})
        got = torch.autograd.grad(loss, list(leaves.values()), allow_unused=True)
        grads = {k: torch.zeros_like(v) if g is None else g
                 for (k, v), g in zip(leaves.items(), got)}
        return h_ref, u, grads

    def check(self):
        h, u = self.forward()
        h_ref, u_ref, grads = self.reference(h)
        _close(h, h_ref, "h")
        if self.pre:
            _close(u, u_ref, "u")
        got = self.backward(h)
        assert set(got) == set(grads), (sorted(got), sorted(grads))
        for k, v in grads.items():
            _close(got[k], v, k)


RAGGED = [0, 1, 1, 38, 60]  # of 70 rows: one row, none, many, many, then padding


@pytest.mark.parametrize("dtype,stream", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("channels", [8, 64, 136, 256, 264, 520, 1408, 2048, 2056, 8192])
def test_sizes(channels, dtype, stream):
    log(f"case norm {channels} {dtype} {stream}")
    Case(70, channels, RAGGED, dtype=dtype, stream=stream).check()


@pytest.mark.parametrize("pre,post", [("layer", None), ("rms", None), ("layer", "rms"),
                                      ("rms", "layer"), (None, None), (None, "rms"),
                                      (None, "layer")])
@pytest.mark.parametrize("channels", [72, 768, 4096])
def test_kinds(channels, pre, post):
    log(f"case norm {channels} {pre} {post}")
    Case(70, channels, RAGGED, pre=pre, post=post).check()


@pytest.mark.parametrize("conds,affine", [("", False), ("", True), ("g", False), ("sf", False),
                                          ("s", True), ("gf", True)])
def test_parameters_that_are_left_out(conds, affine):
    Case(37, 320, [0, 5, 37], conds=conds, affine=affine, post="rms").check()


@pytest.mark.parametrize("pre", ["layer", "rms"])
@pytest.mark.parametrize("off", [None, [0, 12, 30]])
def test_without_branch(pre, off):
    """The first norm of a model: h is x, and only u is written."""
    c = Case(33, 328, off, pre=pre, branch=False)
    h, u = c.forward()
    _, u_ref, grads = c.reference(c.x)
    _close(u, u_ref, "u")
    got = c.plan.backward(c.du.cuda(), c.x.cuda(), **c.dev)  # no dh either
    c.dh = torch.zeros_like(c.dh)
    for k, v in c.reference(c.x)[2].items():
        _close(got[k], v, k)


@pytest.mark.parametrize("tokens,off", [
    (1, None), (1, [0, 0, 1, 1]), (2, [0, 0, 0]), (4, [0, 1, 2, 3, 4]), (1200, None),
    (1200, [0, 599, 600, 1199]), (513, list(range(0, 514, 3)) + [513]), (9, [0, 0]),
    (1025, [0, 1024]),
])
@pytest.mark.parametrize("channels", [64, 768, 2560])
def test_documents(channels, tokens, off):
    log(f"case norm documents {channels} {tokens}")
    Case(tokens, channels, off, post="rms").check()


@pytest.mark.parametrize("channels", [64, 328, 1408])
@pytest.mark.parametrize("tokens,off", [
    (4099, [0, 1, 2, 7, 1000, 1001, 4000, 4000, 4090]), (8195, [0, 3, 5, 4097, 8191, 8194]),
    (8200, None), (5003, list(range(5001))),
])
def test_many_rows(channels, tokens, off):
    """Where a group of lanes takes several rows in order, across documents and
    into the padding; and more documents than one look at 64 offsets finds.  Sums run
    over up to 8200 rows, 11 in a row per block and 768 blocks: as in the rest."""
    log(f"case norm many rows {channels} {tokens}")
    Case(tokens, channels, off, post="rms" if channels == 328 else None).check()


def test_no_tokens():
    c = Case(0, 64, [0, 0, 0])
    h, u = c.forward()
    assert h.shape == u.shape == (0, 64)
    got = c.backward(h)
    assert all(float(got[k].abs().sum()) == 0 for k in got)


def test_gradient_against_differences():
    """d loss / d x along a direction, by central differences of the kernel's
    own fp32 forward.  The difference's truncation is h^2 times the third
    derivative, its rounding 2^-24 of the loss's terms over h: with h = 1e-2 and 64
    x 40 terms of order 1, both below 1e-3 of the sum."""
    c = Case(40, 64, [0, 17, 40], pre="layer", post="rms", dtype=F32, stream=F32)
    h0, _ = c.forward()
    got = c.backward(h0)
    g = torch.Generator().manual_seed(5)
    for name, grad in (("x", "dx"), ("y", "dy")):
        keep, way = getattr(c, name), torch.randn(40, 64, generator=g)
        loss = []
        for s in (1e-2, -1e-2):
            setattr(c, name, keep + s * way)
            h, u = c.forward()
            loss.append(float((h.double().cpu() * c.dh.double()).sum() +
                              (u.double().cpu() * c.du.double()).sum()))
        setattr(c, name, keep)
        want = float((got[grad].double().cpu() * way.double()).sum())
        size = float((got[grad].double().cpu().abs() * way.double().abs()).sum())
        assert abs((loss[0] - loss[1]) / 2e-2 - want) <= 2e-3 * size


def test_padding_takes_no_part():
    """NaN and infinities behind the last document reach nothing but h there."""
    c = Case(50, 136, [0, 20, 31], post="layer")
    clean_h, clean_u = c.forward()
    clean = c.backward(clean_h)
    for name in ("y", "du"):
        getattr(c, name)[31:40] = float("nan")
        getattr(c, name)[40:] = float("inf")
    c.x[33:] = float("nan")
    h, u = c.forward()
    assert torch.equal(h[:31], clean_h[:31]) and torch.equal(u, clean_u)
    assert bool((u[31:] == 0).all())
    assert torch.equal(h[31:].nan_to_num(7), c.x[31:].cuda().nan_to_num(7))
    got = c.backward(h)
    for k in got:
        assert torch.equal(got[k], clean[k]), k
    assert torch.equal(got["dx"][31:], c.dh[31:].cuda()) and bool((got["dy"][31:] == 0).all())


def test_nan_stays_in_its_row_and_document():
    c = Case(20, 72, [0, 8, 20])
    c.y[3, 5] = float("nan")
    h, u = c.forward()
    bad = torch.isnan(u).any(1).cpu()
    assert bad.tolist() == [i == 3 for i in range(20)]
    got = c.backward(h)
    assert bool(torch.isnan(got["dscale"][0]).any())
    assert not bool(torch.isnan(got["dscale"][1]).any())
    assert torch.isnan(got["dx"]).any(1).cpu().tolist() == [i == 3 for i in range(20)]


def test_strides_and_in_place():
    """The tensors inside wider ones, the conditions side by side, h into x and u
    into y, dx into dh and dy into du: the same bits as apart."""
    c = Case(45, 320, [0, 11, 40], dtype=BF, stream=BF)
    want_h, want_u = c.forward()
    want = c.backward(want_h)
    cond = torch.zeros(2, 3 * 320 + 4, device="cuda")
    for i, k in enumerate(("gate", "scale", "shift")):
        cond[:, 320 * i:320 * (i + 1)] = c.dev[k]
        c.dev[k] = cond[:, 320 * i:320 * (i + 1)]
    box = torch.full((45, 5 * 320 + 8), 3.0, dtype=BF, device="cuda")
    x, y, du, dh = (box[:, 320 * i:320 * i + 320] for i in range(4))
    x.copy_(c.x), y.copy_(c.y), du.copy_(c.du), dh.copy_(c.dh)
    keep_y = y.clone()
    h, u = c.plan.forward(x, y, **c.dev, out=(x, y))
    assert torch.equal(h, want_h) and torch.equal(u, want_u) and h.data_ptr() == x.data_ptr()
    assert torch.equal(du, c.du.cuda()) and bool((box[:, 4 * 320:] == 3).all())
    got = c.plan.backward(du, h, dh=dh, y=keep_y, **c.dev, out={"dx": dh, "dy": du})
    for k in got:
        assert torch.equal(got[k], want[k]), k
    assert bool((box[:, 4 * 320:] == 3).all())


def test_rows_far_apart():
    """Offsets above 2^31 elements."""
    far = 1200000000 // 8 * 8
    box = torch.empty(2 * far + 64, dtype=BF, device="cuda")
    c = Case(3, 64, [0, 1, 3], stream=BF)
    want_h, want_u = c.forward()
    x = box.as_strided((3, 64), (far, 1))
    x.copy_(c.x)
    h, u = c.plan.forward(x, c.cuda("y"), **c.dev, out=(x, None))
    assert torch.equal(h, want_h) and torch.equal(u, want_u)


def test_large_values():
    """Rows of 1e18: squares overflow fp32 only above 1.8e19."""
    c = Case(9, 264, None, dtype=F32, stream=F32, conds="", affine=False)
    c.x *= 1e18
    c.y *= 1e18
    c.check()
    z = Case(9, 264, None, dtype=F32, stream=F32, conds="", affine=False, eps=1e-6)
    z.x.zero_(), z.y.zero_()
    h, u = z.forward()
    assert bool((u == 0).all())  # eps keeps rows of zeros finite


def test_streams_and_graph():
    c = Case(200, 768, [0, 64, 150])
    h, u = c.forward()
    want = c.backward(h)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    h2, u2 = c.forward(stream=s)
    got = c.backward(h2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(u, u2) and all(torch.equal(got[k], want[k]) for k in want)
    x, y, du, dh = (c.cuda(k) for k in ("x", "y", "du", "dh"))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hg, ug = c.plan.forward(x, y, **c.dev)
        got = c.plan.backward(du, hg, dh=dh, y=y, **c.dev)
    for i in range(3):
        if i:
            x.mul_(1.5), du.add_(0.25)
            c.x, c.du = x.cpu(), du.cpu()
        g.replay()
        torch.cuda.synchronize()
        h, u = c.forward()
        want = c.backward(h)
        assert torch.equal(hg, h) and torch.equal(ug, u)
        for k in want:
            assert torch.equal(got[k], want[k]), (i, k)
