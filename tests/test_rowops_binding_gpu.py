"""The binding of the row operators: what it refuses, memory on other streams,
and calls from two threads on one object."""

import threading

import pytest
import torch

from paper_2606_19163_amd import ops
from paper_2606_19163_amd.stage import PulseError

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _rows(t, c, dtype=BF):
    return torch.randn(t, c, device="cuda").to(dtype)


def _refused(what, fn):
    with pytest.raises(PulseError, match=what):
        fn()


def test_norm_refuses():
    n = ops.Norm(64, docs=2)
    off = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    x, y, cond = _rows(5, 64), _rows(5, 64), torch.zeros(2, 64, device="cuda")
    _refused("y is missing", lambda: n.forward(x, offsets=off))
    _refused("x is", lambda: n.forward(_rows(5, 72), y, offsets=off))
    _refused("x is", lambda: n.forward(x.float(), y, offsets=off))
    _refused("contiguous", lambda: n.forward(_rows(64, 5).t(), y, offsets=off))
    _refused("current GPU", lambda: n.forward(x.cpu(), y, offsets=off))
    _refused("offsets", lambda: n.forward(x, y, offsets=off[:2]))
    _refused("offsets", lambda: n.forward(x, y, offsets=off.long()))
    _refused("offsets is NULL", lambda: n.forward(x, y))
    _refused("gate", lambda: n.forward(x, y, offsets=off, gate=cond[:1]))
    _refused("scale", lambda: n.forward(x, y, offsets=off, scale=cond.to(BF)))
    _refused("shift", lambda: n.forward(x, y, offsets=off, shift=cond[0]))
    _refused("weight", lambda: n.forward(x, y, offsets=off, weight=cond[0].cpu()))
    _refused("no use", lambda: n.forward(x, y, offsets=off, post_weight=cond[0].clone()))
    _refused("overlaps", lambda: n.forward(x, y, offsets=off, out=(None, x)))
    _refused("is missing", lambda: n.backward(None, x, y=y, offsets=off))
    _refused("does not compute", lambda: n.backward(x, y, y=y, offsets=off, out={"dgate": cond}))
    _refused("dx is", lambda: n.backward(x, y, y=y, offsets=off, out={"dx": _rows(4, 64)}))
    only = ops.Norm(64, pre=None)
    _refused("is given", lambda: only.backward(x, None, y=y))
    assert n.forward(x[:0], y[:0], offsets=off)[1].shape == (0, 64)


def test_checkpoint_refuses():
    c = ops.Checkpoint(64)
    x = _rows(6, 64)
    kept = c.save(x)
    _refused("holds nothing", lambda: c.load(c.buffer(6)))
    _refused("is of 6 tokens", lambda: c.weight_grad(_rows(5, 16), kept))
    _refused("is of 6 tokens", lambda: ops.Checkpoint(72).load(kept))
    _refused("no act", lambda: c.forward(x))
    _refused("no act", lambda: c.save(x, out=_rows(6, 64)))
    _refused("no act", lambda: c.backward(x, kept))
    _refused("out is None", lambda: c.weight_grad(_rows(6, 16), kept, accumulate=True))
    _refused("out is", lambda: c.weight_grad(_rows(6, 16), kept, out=torch.empty(64, 16).cuda()))
    _refused("dy is", lambda: c.weight_grad(_rows(6, 16, torch.float32), kept))
    _refused("multiple of 8", lambda: c.weight_grad(_rows(6, 20)[:, :12], kept))
    g = ops.Checkpoint(64, act="gelu")
    _refused("overlaps", lambda: g.backward(x, kept, again=kept))


def test_linear8_refuses():
    w = torch.randn(24, 64, device="cuda")
    _refused("inputs and outputs", lambda: ops.Linear8(w[:, :60].contiguous()))
    _refused("contiguous", lambda: ops.Linear8(torch.randn(64, 24, device="cuda").t()))
    _refused("dtype", lambda: ops.Linear8(w.half()))
    _refused("bias", lambda: ops.Linear8(w, bias=torch.zeros(16, device="cuda")))
    layer = ops.Linear8(w)
    _refused("weight is", lambda: layer.update(w[:16].contiguous()))
    _refused("x is", lambda: layer.forward(_rows(3, 72)))
    _refused("x is", lambda: layer.forward(_rows(3, 64, torch.float32)))
    _refused("out is", lambda: layer.forward(_rows(3, 64), out=_rows(3, 32)))
    _refused("current GPU", lambda: layer.forward(_rows(3, 64).cpu()))


def test_autograd_is_refused_but_under_no_grad():
    x = _rows(4, 64).requires_grad_(True)
    w = torch.randn(24, 64, device="cuda", requires_grad=True)
    n, c, g = ops.Norm(64), ops.Checkpoint(64), ops.Checkpoint(64, act="silu")
    y = _rows(4, 64)
    for fn in (lambda: n.forward(x, y), lambda: n.forward(y, x), lambda: c.save(x),
               lambda: g.forward(x), lambda: ops.Linear8(w),
               lambda: ops.Linear8(w.detach()).forward(x),
               lambda: n.forward(y, y, weight=torch.ones(64, device="cuda", requires_grad=True))):
        _refused("requires a gradient", fn)
        with torch.no_grad():
            fn()


def test_memory_on_another_stream():
    """Objects dropped while another stream still works on their memory."""
    s = torch.cuda.Stream()
    x = _rows(4096, 1408)
    layer = ops.Linear8(torch.randn(1408, 1408, device="cuda"), bias=torch.randn(1408).cuda())
    kept = ops.Checkpoint(1408).save(x)
    want = layer.forward(x), ops.Checkpoint(1408).load(kept)
    torch.cuda.synchronize()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(20):
        outs.append(layer.forward(x, stream=s))
    back = ops.Checkpoint(1408).load(kept, stream=s)
    del layer, kept
    junk = [torch.full((4 << 20,), float("nan"), device="cuda") for _ in range(16)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) for o in outs) and torch.equal(back, want[1])
    del junk


def test_two_threads_on_one_object():
    """Calls at once on two streams share no workspace."""
    t, c = 700, 768
    layer = ops.Linear8(torch.randn(1000, c, device="cuda"))
    norm, keep = ops.Norm(c), ops.Checkpoint(c)
    ins = [(_rows(t, c), _rows(t, c), _rows(t, 1000)) for _ in range(2)]

    def work(i, out):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.default_stream())
        x, y, dy = ins[i]
        w = torch.ones(c, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(30):
                h, u = norm.forward(x, y, weight=w)
                grads = norm.backward(y, h, y=y, weight=w)
                out[i] = [layer.forward(u), keep.weight_grad(dy, keep.save(u)), grads["dweight"],
                          grads["dx"]]
        s.synchronize()

    alone, both = {}, {}
    for i in range(2):
        work(i, alone)
    ts = [threading.Thread(target=work, args=(i, both)) for i in range(2)]
    for th in ts:
        th.start()
    for th in ts:
        th.join()
    for i in range(2):
        for a, b in zip(alone[i], both[i]):
            assert torch.equal(a, b), i
