"""Integer sums of the 8-bit linear layers, exactly: the inputs are whole numbers whose
rows have a largest value of 127, so that they are kept as they are with a scale of 1 (or
of 254: halves are ties, and the scale is 2), and results are compared for equality."""

import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

#: tokens, inputs, outputs: a token that every block lays out for itself, few tokens, a
#: tile of 64 x 64, of 64 x 128, of 128 x 256
PATHS = [(1, 32000, 64), (3, 10504, 24), (16, 65536, 40), (33, 65536, 24), (64, 20008, 136),
         (70, 65536, 40), (300, 8192, 136), (2048, 4096, 2056), (4096, 4096, 2048)]


@pytest.mark.parametrize("tokens,inputs,outputs", PATHS)
def test_large_sums_that_cancel(tokens, inputs, outputs):
    """Half of the products are 127 * 127 and half -127 * 127, among them eight small ones,
    which alone are left: partial sums pass 2^24 (but for the first case), where fp32
    would lose them, and the results, of at most 8 * 5 * 6 = 240, are exact in bf16."""
    log(f"case lin8 cancel {tokens}x{inputs}->{outputs}")
    g = torch.Generator().manual_seed(inputs)
    half = inputs // 2
    x, w = torch.full((tokens, inputs), 127.0), torch.full((outputs, inputs), 127.0)
    w[:, half:] = -127.0
    # as many of either sign, wherever the small ones are
    at = torch.cat([torch.randperm(half - 1, generator=g)[:4],
                    half + torch.randperm(half - 1, generator=g)[:4]])
    x[:, at] = torch.randint(-5, 6, (tokens, 8), generator=g).float()
    w[:, at] = torch.randint(-6, 7, (outputs, 8), generator=g).float()
    want = x[:, at] @ w[:, at].t()
    flip = torch.randint(0, 2, (inputs,), generator=g).float() * 2 - 1  # any order of signs
    x, w = x * flip, w * flip
    y = ops.Linear8(w.cuda()).forward(x.to(BF).cuda())
    assert torch.equal(y.cpu().float(), want)


@pytest.mark.parametrize("tokens", [1, 16, 40, 300, 2100])
def test_ties_go_to_even(tokens):
    """The factor is the quotient 127 / 254, exactly 1 / 2: odd numbers are ties."""
    g = torch.Generator().manual_seed(tokens)
    n = 4096 if tokens > 1000 else 72
    x = torch.randint(-254, 255, (tokens, 520), generator=g).float()
    w = torch.randint(-254, 255, (n, 520), generator=g).float()
    x[:, 7], w[:, 11] = 254, -254

    def even(v):
        v = v.to(BF).float()
        v = torch.where(v.abs() > 254, v.sign() * 254, v)
        low = torch.floor(v / 2)
        tie = v / 2 != low
        return torch.where(tie, low + (low % 2 != 0), low)

    y = ops.Linear8(w.to(BF).cuda()).forward(x.to(BF).cuda()).cpu()
    want = 4 * (even(x).double() @ even(w).double().t())
    assert float(want.abs().max()) < 2 ** 24  # exact in fp32, then rounded once
    assert torch.equal(y, want.float().to(BF))
