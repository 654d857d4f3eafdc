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
