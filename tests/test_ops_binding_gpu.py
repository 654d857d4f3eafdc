"""How the operators' binding allocates and what it takes, on a GPU."""

import pytest
import torch

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _mask(*off):
    m = ops.Mask(off[-1], docs=len(off) - 1)
    m.build(torch.tensor(off, dtype=torch.int32, device="cuda"))
    return m


def test_tensors_that_require_a_gradient():
    q = torch.randn(70, 2, 64, device="cuda").to(BF).requires_grad_()
    pos, freq = torch.zeros(70, 1, device="cuda"), ops.rope_freqs([64])
    plan, rope, m = ops.Attn(70, 2, 64), ops.Rope(2, 64, [64]), _mask(0, 70)
    for call in (lambda: plan.forward(q, q, q, m), lambda: rope.forward(q, pos, freq)):
        with pytest.raises(S.PulseError, match="requires a gradient"):
            call()
        with torch.no_grad():
            call()
    d = q.detach()
    o, saved = plan.forward(d, d, d, m)
    with torch.no_grad():
        p, _ = plan.forward(q, q, q, m)
    assert torch.equal(o, p)
    dq, _, _ = plan.backward(d, d, d, d, o, saved, m)
    assert torch.isfinite(dq).all()


@pytest.mark.parametrize("queries,keys,dim", [(300, 300, 64), (300, 300, 128), (3, 6000, 88)])
def test_forward_that_keeps_nothing(queries, keys, dim):
    """The same output; of a step's memory, the output, lse and the workspace."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    q = torch.randn(queries, 8, dim, generator=g, device="cuda").to(BF)
    k, v = (torch.randn(keys, 8, dim, generator=g, device="cuda").to(BF) for _ in range(2))
    m = ops.Mask(queries, keys=keys, docs=1)
    m.build(torch.tensor([0, queries], dtype=torch.int32, device="cuda"),
            key_offsets=torch.tensor([0, keys], dtype=torch.int32, device="cuda"))
    plan = ops.Attn(queries, 8, dim, keys=keys)
    want, saved = plan.forward(q, k, v, m)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    o, none = plan.forward(q, k, v, m, keep=False)
    used = torch.cuda.max_memory_allocated() - before
    assert none is None and torch.equal(o, want)
    parts = [2 * o.numel(), 4 * 8 * queries, plan.fwd_bytes]
    assert used <= sum(-(-p // 512) * 512 for p in parts)  # the allocator's blocks
    with pytest.raises(S.PulseError, match="nothing is to be kept"):
        plan.forward(q, k, v, m, saved=saved, keep=False)


@pytest.mark.parametrize("what", ["mask", "saved", "clip"])
def test_memory_of_objects_used_on_another_stream(what):
    """It is not handed on while that stream has work with it ahead."""
    t = 2048
    q = torch.randn(t, 4, 64, device="cuda").to(BF)
    off = torch.tensor([0, t], dtype=torch.int32, device="cuda")
    plan = ops.Attn(t, 4, 64)
    side = torch.cuda.Stream()
    keep = _mask(0, t)
    o, s0 = plan.forward(q, q, q, keep)
    out = [torch.empty_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = {"mask": ops.Mask(t, docs=1), "saved": ops.Saved(4, t, 64, "cuda"),
            "clip": ops.GradClip([torch.ones(1 << 20, device="cuda")])}
    held["mask"].build(off)
    plan.forward(q, q, q, keep, saved=held["saved"])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    if what == "mask":
        plan.forward(q, q, q, held["mask"], out=out[0], saved=s0, stream=side)
        s0.mask = None  # it would keep the mask
    elif what == "saved":
        plan.backward(q, q, q, q, o, held["saved"], keep, out=out, stream=side)
    else:
        norm = torch.empty(1, device="cuda")
        held["clip"].run(1.0, norm=norm, stream=side)
    busy = not side.query()
    x = held.pop(what)
    buf = x.workspace if what == "clip" else x.buffer
    ptr, numel = buf.data_ptr(), buf.numel() * buf.element_size()
    del x, buf
    again = torch.empty(numel, dtype=torch.uint8, device="cuda").data_ptr()
    torch.cuda.synchronize()
    assert busy and again != ptr


@pytest.mark.parametrize("queries,keys", [(0, 0), (0, 70), (5, 0), (200, 0), (0, 5000)])
@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 1)])
def test_attn_without_rows_or_keys(queries, keys, heads, kv):
    """Every output that there is, is 0."""
    m = ops.Mask(queries, keys=keys, docs=1)
    m.build(torch.tensor([0, queries], dtype=torch.int32, device="cuda"),
            key_offsets=torch.tensor([0, keys], dtype=torch.int32, device="cuda"))
    plan = ops.Attn(queries, heads, 64, keys=keys, kv_heads=kv)
    q, k = torch.ones(plan.qs, device="cuda").to(BF), torch.ones(plan.ks, device="cuda").to(BF)
    o, saved = plan.forward(q, k, k, m)
    out = [torch.full_like(x, 7.0) for x in (q, k, k)]
    plan.backward(q, q, k, k, o, saved, m, out=out)
    assert (saved.lse == -float("inf")).all()
    for x in (o, *out):
        assert (x == 0).all()


def test_clip_refuses_tensors_that_overlap():
    x = torch.ones(100, device="cuda")
    for grads, outs in (([x, x], None), ([x[:60], x[50:]], None), ([x[:50]], [x[1:51]])):
        with pytest.raises(S.PulseError, match="overlaps"):
            ops.GradClip(grads, outs)
    y = torch.empty(200, device="cuda")
    n = ops.GradClip([x, x], [y[:100], y[100:]]).run(1.0)  # read twice, written apart
    assert abs(float(n) - 200 ** 0.5) <= 1e-5


def test_clip_runs_at_once_on_any_stream():
    """The tensors' table is there when the object is: behind work that the
    stream it was made on still has ahead, and without an event between."""
    side = torch.cuda.Stream()
    x = torch.ones(1 << 20, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    clip = ops.GradClip([x])
    assert torch.cuda.current_stream().query()
    n = clip.run(512.0, stream=side)
    side.synchronize()
    assert abs(float(n) - 1024.0) <= 1e-3 and abs(float(x[0]) - 0.5) <= 1e-6
