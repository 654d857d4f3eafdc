"""Inputs that require a gradient are refused where torch would record one,
not cut from it silently (no GPU: refused before any is looked for)."""

import pytest
import torch

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import built  # noqa: F401  (builds the library)

BF = torch.bfloat16


def _grad(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype, requires_grad=True)


@pytest.mark.parametrize("name", ["x", "pos", "freq"])
def test_rope(name):
    args = dict(x=torch.zeros(5, 2, 64, dtype=BF), pos=torch.zeros(5, 1), freq=torch.zeros(32))
    args[name] = args[name].requires_grad_()
    with pytest.raises(S.PulseError, match=f"{name} requires a gradient"):
        ops.Rope(2, 64, [64]).forward(**args)
    # a product of such a tensor is one too
    if name == "x":
        args["x"] = args["x"] * 2
        with pytest.raises(S.PulseError, match="x requires a gradient"):
            ops.Rope(2, 64, [64]).forward(**args)


@pytest.mark.parametrize("name", ["q", "k", "v", "slopes"])
def test_attn(name):
    args = {n: torch.zeros(5, 2, 64, dtype=BF) for n in ("q", "k", "v")}
    args["slopes"] = torch.zeros(2)
    args[name] = args[name].requires_grad_()
    mask = ops.Mask(5, docs=1, device="cpu")
    mask._built()
    with pytest.raises(S.PulseError, match=f"{name} requires a gradient"):
        ops.Attn(5, 2, 64).forward(mask=mask, **args)


def test_by_hand_under_no_grad():
    """There is nothing to refuse (what is missing then is the GPU)."""
    for ctx in (torch.no_grad(), torch.inference_mode()):
        with ctx:
            assert not ops._grad_on()
    ops._by_hand(("x", _grad(3).detach()), ("y", None))


def test_gradients_of_gradients():
    with pytest.raises(S.PulseError, match="dout requires a gradient"):
        ops.Rope(2, 64, [64]).backward(_grad(5, 2, 64), torch.zeros(5, 1), torch.zeros(32))
    t, m = torch.zeros(5, 2, 64, dtype=BF), ops.Mask(5, docs=1, device="cpu")
    with pytest.raises(S.PulseError, match="dout requires a gradient"):
        ops.Attn(5, 2, 64).backward(_grad(5, 2, 64), t, t, t, t, ops.Saved(2, 5, 64, "cpu"), m)
