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
