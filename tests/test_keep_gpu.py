"""Activations kept in 8 bits: what is kept against the definition, value for
value, and what is computed from it against float64 forms.

Tolerances.  Kept values are equal to the definition's.  act(x) and the gradient
are computed in fp32 and rounded once: half a step (2^-8 of the value in bf16,
2^-24 in fp32), and the activation's own error, 3e-7 (1 + |z|) where erf is
taken from a formula with an error of 1.5e-7, times the incoming gradient.  The
weight gradient's products are exact, and a sum of T of them in fp32 is off by
at most T 2^-24 of the sum of their sizes; roundings have either sign, so about
sqrt(T) 2^-24 of the result in the L2 norm: 1e-5 covers T = 8192 (5.4e-6)."""

import math

import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log, rel_l2

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=F32)


def _kept_ref(x):
    """The definition, group by group: (values in float64, steps)."""
    t, c = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -c % 32)).reshape(-1, 32)
    out, steps = torch.empty_like(v), torch.empty(v.shape[0], dtype=torch.float64)
    for i, row in enumerate(v):
        top = float(row.abs().max())
        if not math.isfinite(top):
            out[i], steps[i] = float("nan"), float("nan")
            continue
        e = -126
        if top > 0:
            e = max(e, math.frexp(top)[1] - 8)
        while e < 121 and float(torch.round(torch.tensor(top / 2.0 ** e,
                                                         dtype=torch.float64))) > 127:
            e += 1
        out[i] = torch.round(row / 2.0 ** e).clamp(-127, 127) * 2.0 ** e
        steps[i] = 2.0 ** e
    return (out.reshape(t, -1)[:, :c],
            steps.reshape(t, -1).repeat_interleave(32, 1)[:, :c])


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z * torch.sigmoid(z)


def _act_grad(z, act):
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(_act(z, act).sum(), z)[0]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,channels", [(1, 8), (3, 40), (5, 320), (130, 32), (2, 1408),
                                             (7, 4104), (67, 264), (1, 65536)])
def test_kept_values(tokens, channels, dtype):
    log(f"case keep {tokens}x{channels} {dtype}")
    x = (_randn(tokens + channels, tokens, channels) *
         torch.exp(1.5 * _randn(1, channels))).to(dtype)
    plan = ops.Checkpoint(channels, dtype=dtype)
    got = plan.load(plan.save(x.cuda())).cpu().double()
    ref, step = _kept_ref(x)
    assert torch.equal(got, ref)
    assert bool(((got - x.double()).abs() <= 0.5 * step).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_kept_edges(dtype):
    """Ties, the border of a power of two (127.5 rounds to 128, so that it needs
    the next one), zeros, the smallest and the largest values, NaN and inf."""
    top = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).tiny
    rows = [torch.zeros(32), torch.full((32,), -0.0), torch.full((32,), top),
            torch.full((32,), -top), torch.full((32,), tiny), torch.full((32,), tiny / 64),
            torch.arange(32) * 0.5 + 64.5, torch.arange(32) * 0.5 - 127.5,
            torch.arange(32) - 127.0, torch.full((32,), 1.9921875), torch.full((32,), 1.984375),
            torch.full((32,), 2.0 ** -119), torch.full((32,), 255 * 2.0 ** -127)]
    x = torch.stack(rows).to(dtype)
    for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
        x = torch.cat([x, _randn(i, 1, 32).to(dtype)])
        x[-1, 7 * i] = bad
    x = torch.cat([x, _randn(9, x.shape[0], 32).to(dtype)], dim=1)  # a sound group beside it
    plan = ops.Checkpoint(64, dtype=dtype)
    got = plan.load(plan.save(x.cuda())).cpu().double()
    ref, _ = _kept_ref(x)
    assert torch.equal(got.nan_to_num(12345.0), ref.nan_to_num(12345.0))
    assert not bool(torch.isnan(got[:, 32:]).any())


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,channels", [(1, 8), (33, 136), (70, 1024), (6, 5632)])
def test_activation(tokens, channels, dtype, act):
    log(f"case keep {act} {tokens}x{channels} {dtype}")
    x = (3 * _randn(channels, tokens, channels)).to(dtype)
    da = _randn(7, tokens, channels).to(dtype)
    plan = ops.Checkpoint(channels, act=act, dtype=dtype)
    a, kept = plan.forward(x.cuda())
    z, _ = _kept_ref(x)
    assert torch.equal(plan.load(kept).cpu().double(), z)
    again = plan.buffer(tokens)
    dx = plan.backward(da.cuda(), kept, again=again)
    assert torch.equal(dx, plan.backward(da.cuda(), kept))
    half = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    for got, ref, size in ((a, _act(x.double(), act), 1 + x.double().abs()),
                           (dx, da.double() * _act_grad(z, act),
                            da.double().abs() * (1 + z.abs()))):
        off = (got.cpu().double() - ref).abs()
        assert bool((off <= half * ref.abs() + 3e-7 * size).all())
    # kept again: within half a step, which is at most 1 / 127 of the group's largest
    want = _act(z, act)
    got = plan.load(again).cpu().double()
    pad = torch.nn.functional.pad(want, (0, -channels % 32)).reshape(tokens, -1, 32)
    top = pad.abs().amax(2).repeat_interleave(32, 1)[:, :channels]
    assert bool(((got - want).abs() <= 1.001 * top / 127 + 3e-7 * (1 + z.abs())).all())


def test_activation_of_infinities_and_nan():
    x = torch.zeros(4, 64, dtype=BF)
    x[0, 0], x[1, 0], x[2, 0] = float("nan"), float("inf"), -30.0
    plan = ops.Checkpoint(64, act="gelu")
    a, kept = plan.forward(x.cuda())
    assert bool(torch.isnan(a[0, 0])) and float(a[1, 0]) == float("inf") and float(a[2, 0]) == 0
    dx = plan.backward(torch.ones_like(x).cuda(), kept)
    assert torch.isnan(dx).sum(1).tolist() == [32, 32, 0, 0]


def test_strides_and_in_place():
    t, c = 41, 328
    box = torch.full((t, 2 * c + 8), 5.0, dtype=BF, device="cuda")
    x, d = box[:, :c], box[:, c:2 * c]
    x.copy_(_randn(1, t, c)), d.copy_(_randn(2, t, c))
    plan = ops.Checkpoint(c, act="silu")
    a, kept = plan.forward(x)
    dx = plan.backward(d, kept)
    z = plan.load(kept)
    other = plan.save(x, out=x)
    assert torch.equal(x, a) and torch.equal(plan.load(other), z)
    assert torch.equal(plan.backward(d, kept, out=d), dx)
    plan.load(kept, out=x)
    assert torch.equal(x, z) and torch.equal(d, dx) and bool((box[:, 2 * c:] == 5).all())
    far = 1200000000 // 8 * 8  # offsets above 2^31 elements
    big = torch.empty(2 * far + 64, dtype=BF, device="cuda").as_strided((3, 64), (far, 1))
    big.copy_(_randn(3, 3, 64))
    plan = ops.Checkpoint(64)
    ref = plan.load(plan.save(big.contiguous()))
    assert torch.equal(plan.load(plan.save(big), out=big), ref)


# ---- weight gradients ------------------------------------------------------------


def _wgrad(tokens, channels, outputs, bias=True, accumulate=False, seed=0):
    x = (_randn(seed + 1, tokens, channels) * torch.exp(_randn(seed + 2, channels))).to(BF)
    dy = _randn(seed + 3, tokens, outputs).to(BF)
    plan = ops.Checkpoint(channels)
    kept = plan.save(x.cuda())
    xk = plan.load(kept).double()
    dw = torch.full((outputs, channels), 3.0, device="cuda")
    db = torch.full((outputs,), -2.0, device="cuda") if bias else None
    got = plan.weight_grad(dy.cuda(), kept, out=dw, bias_out=db, accumulate=accumulate)
    assert got.data_ptr() == dw.data_ptr()
    d64 = dy.cuda().double()
    ref = d64.t().contiguous() @ xk + (3.0 if accumulate else 0.0)
    assert rel_l2(dw.double().cpu(), ref.cpu()) <= 1e-5
    # per value: T roundings of its sum of sizes, and the sum with what was there
    size = d64.abs().t().contiguous() @ xk.abs() + 3.0
    assert bool(((dw.double() - ref).abs() <= (tokens + 1) * 2.0 ** -24 * size).all())
    if bias:
        refb = d64.sum(0) - (2.0 if accumulate else 0.0)
        assert bool(((db.double() - refb).abs() <=
                     (tokens + 1) * 2.0 ** -24 * (d64.abs().sum(0) + 2)).all())


@pytest.mark.parametrize("tokens,channels,outputs", [
    (1, 8, 8), (63, 40, 72), (64, 64, 64), (65, 136, 8), (1000, 320, 200), (3, 1408, 264),
    (2747, 320, 1280), (200, 8, 1024), (130, 264, 520),
])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad(tokens, channels, outputs, accumulate):
    log(f"case wgrad {tokens}x{channels}->{outputs} {accumulate}")
    _wgrad(tokens, channels, outputs, accumulate=accumulate)


@pytest.mark.parametrize("tokens,channels,outputs", [
    (8192, 1024, 1032), (4100, 1416, 2056), (1025, 2048, 4096), (5000, 1000, 1000),
])
@pytest.mark.parametrize("bias", [False, True])
def test_weight_grad_of_many(tokens, channels, outputs, bias):
    log(f"case wgrad {tokens}x{channels}->{outputs} {bias}")
    _wgrad(tokens, channels, outputs, bias=bias)
    _wgrad(tokens, channels, outputs, bias=bias, accumulate=True)


@pytest.mark.parametrize("tokens,channels,outputs", [
    (4100, 6000, 40), (9000, 64, 6008), (10000, 136, 136), (70000, 64, 64),
])
def test_weight_grad_of_a_narrow_axis(tokens, channels, outputs):
    """Many partial sums of one value: more than eight of dw, more than 128 of db."""
    log(f"case wgrad {tokens}x{channels}->{outputs}")
    _wgrad(tokens, channels, outputs)
    _wgrad(tokens, channels, outputs, accumulate=True)


def test_weight_grad_in_parts():
    """Tokens whose fragments would take more than 512 MB are taken in parts: 2^28 /
    65536 channels = 4096 at a time, here two of them and 100 tokens."""
    _wgrad(8292, 65536, 8)
    _wgrad(4196, 65536, 136, accumulate=True)


def test_weight_grad_without_tokens():
    plan = ops.Checkpoint(40)
    kept = plan.save(torch.empty(0, 40, dtype=BF, device="cuda"))
    dy = torch.empty(0, 24, dtype=BF, device="cuda")
    db = torch.ones(24, device="cuda")
    dw = plan.weight_grad(dy, kept, bias_out=db)
    assert float(dw.abs().sum()) == 0 and float(db.abs().sum()) == 0
    dw.fill_(2), db.fill_(3)
    plan.weight_grad(dy, kept, out=dw, bias_out=db, accumulate=True)
    assert bool((dw == 2).all()) and bool((db == 3).all())


@pytest.mark.parametrize("tokens,channels,outputs", [(70, 96, 80), (8192, 1024, 1024)])
def test_weight_grad_values_stay_in_their_column(tokens, channels, outputs):
    """A group that is NaN reaches its channels only, an infinite dy its output
    only: not the lanes past the last token."""
    x, dy = _randn(1, tokens, channels).to(BF), _randn(2, tokens, outputs).to(BF)
    x[-1, 40] = float("nan")
    dy[-1, 9] = float("inf")
    plan = ops.Checkpoint(channels)
    db = torch.empty(outputs, device="cuda")
    dw = plan.weight_grad(dy.cuda(), plan.save(x.cuda()), bias_out=db)
    bad = ~torch.isfinite(dw)
    assert bool(bad[:, 32:64].all()) and bool(bad[9].all())
    bad[:, 32:64] = False
    bad[9] = False
    assert not bool(bad.any())
    assert (~torch.isfinite(db)).nonzero().flatten().tolist() == [9]


def test_weight_grad_strided_and_far():
    t, c, n = 190, 72, 88
    box = torch.zeros(t, 3 * n + 8, dtype=BF, device="cuda")
    dy = box[:, n:2 * n]
    dy.copy_(_randn(1, t, n))
    plan = ops.Checkpoint(c)
    kept = plan.save(_randn(2, t, c).to(BF).cuda())
    assert torch.equal(plan.weight_grad(dy, kept), plan.weight_grad(dy.contiguous(), kept))
    far = 1200000000 // 8 * 8
    big = torch.empty(2 * far + n, dtype=BF, device="cuda").as_strided((3, n), (far, 1))
    big.copy_(dy[:3])
    kept = plan.save(_randn(3, 3, c).to(BF).cuda())
    assert torch.equal(plan.weight_grad(big, kept), plan.weight_grad(dy[:3].contiguous(), kept))


def test_streams_and_graph():
    t, c, n = 300, 320, 520
    x, g = _randn(1, t, c).to(BF).cuda(), _randn(2, t, c).to(BF).cuda()
    dy = _randn(3, t, n).to(BF).cuda()
    plan = ops.Checkpoint(c, act="gelu")

    def work(stream=None):
        a, kept = plan.forward(x, stream=stream)
        again = plan.buffer(t)
        dx = plan.backward(g, kept, again=again, stream=stream)
        db = torch.empty(n, device="cuda")
        dw = plan.weight_grad(dy, again, bias_out=db, stream=stream)
        return a, dx, plan.load(again, stream=stream), dw, db

    want = work()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = work(s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for i in range(3):
        if i:
            x.mul_(1.25), dy.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(work(), got)), i


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activation_gradient_against_differences(act):
    """Central differences of the kernel's own fp32 forward around kept values: the
    truncation is below h^2 / 6 times the third derivative (at most 1.6), the
    rounding 6e-7 (1 + |z|) / h; with h = 1e-2 both below 4e-4."""
    plan = ops.Checkpoint(64, act=act, dtype=F32)
    kept = plan.save(2 * _randn(1, 50, 64).cuda())
    z = plan.load(kept)
    got = plan.backward(torch.ones_like(z), kept)
    up, down = (plan.forward(z + s)[0].double() for s in (1e-2, -1e-2))
    assert float(((up - down) / 2e-2 - got.double()).abs().max()) <= 4e-4
