"""Attention scores over the whole range of caps, scales and slopes.

Bounds.  A score z is formed in fp32 from an fp32 product, so it is off by a
few 2^-24 of its size and of what it is a difference of; the capped form adds
at most 1.5e-7 times the cap where |z| is a quarter of the cap or more (one
rounding of exp, of the reciprocal and of their operands), which is at most
1.2e-6 |z|.  lse is within that of the largest |z|, and within 2e-5 where
scores are of unit size.  The outputs' bound is the bf16 operands' (see
test_ops_gpu)."""

import math

import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log, rel_l2
from test_ops_gpu import ATTN_TOL, _attn_check, _attn_ref, _attn_run, _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [0.25, 64.0, 100.0, 1e4, 1e6, 1e8, 1e20, 3e38])
@pytest.mark.parametrize("dim", [64, 88, 128])
def test_attn_caps(dim, cap):
    """A cap far above the scores leaves them as they are."""
    log(f"case attention dim {dim} cap {cap}")
    q, k, v, do, mask, rows = _case([70, 1, 130], 9, 4, 2, dim, "causal", dim)
    slopes = torch.tensor([0.5, 0.05, 0.25, 0.0])
    for sl in (None, slopes):
        plan = ops.Attn(len(rows), 4, dim, kv_heads=2, cap=cap)
        ref = _attn_ref(q, k, v, do, rows, 1 / math.sqrt(dim), cap, sl)
        _attn_check(_attn_run(plan, mask, q, k, v, do, sl), ref, f"cap {cap}")


@pytest.mark.parametrize("cap", [40.0, 100.0, 1000.0, 1e5])
def test_attn_scores_near_and_far_from_the_cap(cap):
    """Some scores near the cap, others of unit size, in one wave's rows."""
    q, k, v, do, mask, rows = _case([200], 0, 2, 2, 64, "doc", 31)
    q = q.float()
    q[::3] *= cap / 4  # scores of about a quarter of the cap
    q = q.to(torch.bfloat16)
    plan = ops.Attn(200, 2, 64, cap=cap)
    ref = _attn_ref(q, k, v, do, rows, 0.125, cap, None)
    got = _attn_run(plan, mask, q, k, v, do)
    far = torch.arange(200) % 3 == 0
    assert (got["lse"] - ref["lse"])[:, ~far].abs().max() <= 2e-5
    assert (got["lse"] - ref["lse"])[:, far].abs().max() <= 2e-5 + 1.2e-6 * cap
    for rowset in (far, ~far):
        assert rel_l2(got["o"][rowset], ref["o"][rowset]) <= ATTN_TOL
    # of the rows whose scores fp32 holds to 1e-5
    assert rel_l2(got["dq"][~far], ref["dq"][~far]) <= ATTN_TOL


def test_attn_cap_below_every_score():
    """Scores of 0 and others under a cap so small that scale / cap overflows."""
    q, k, v, do, mask, rows = _case([90], 6, 2, 2, 64, "causal", 32)
    q[10:20] = 0.0
    plan = ops.Attn(96, 2, 64, cap=1e-40)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 1e-40, None)
    got = _attn_run(plan, mask, q, k, v, do)
    assert (got["lse"] - ref["lse"])[torch.isfinite(ref["lse"])].abs().max() <= 2e-5
    for n in ("o", "dv"):
        assert rel_l2(got[n], ref[n]) <= ATTN_TOL, n


@pytest.mark.parametrize("lens,pad", [([150], 0), ([33, 70, 1], 5), ([129], 0)])
@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-3, -3.0])
@pytest.mark.parametrize("slopes", [None, [0.25, 0.01], [-0.02, -1.5]])
def test_attn_gradient_of_other_scales(scale, slopes, lens, pad):
    """Scales of 0 and below, with slopes of either sign."""
    log(f"case attention scale {scale} slopes {slopes} lengths {lens}")
    sl = None if slopes is None else torch.tensor(slopes)
    for kind in ("doc", "causal"):
        q, k, v, do, mask, rows = _case(lens, pad, 2, 1, 64, kind, 33)
        plan = ops.Attn(len(rows), 2, 64, kv_heads=1, scale=scale)
        ref = _attn_ref(q, k, v, do, rows, scale, 0.0, sl)
        got = _attn_run(plan, mask, q, k, v, do, sl)
        big = max(1.0, ref["lse"][torch.isfinite(ref["lse"])].abs().max())
        live = torch.isfinite(ref["lse"])
        assert (got["lse"] - ref["lse"])[live].abs().max() <= 2e-5 * big
        for n in ("o", "dq", "dk", "dv"):
            if ref[n].abs().sum() > 0:
                assert rel_l2(got[n], ref[n]) <= ATTN_TOL, n
            else:
                assert (got[n] == 0).all(), n


@pytest.mark.parametrize("cap", [2.0, 50.0, 1e4])
@pytest.mark.parametrize("scale", [0.0, -0.125, -1.0])
def test_attn_caps_of_other_scales(scale, cap):
    log(f"case attention scale {scale} cap {cap}")
    q, k, v, do, mask, rows = _case([33, 70, 1], 5, 2, 1, 64, "causal", 34)
    for slopes in (None, torch.tensor([0.25, -0.01])):
        plan = ops.Attn(len(rows), 2, 64, kv_heads=1, scale=scale, cap=cap)
        ref = _attn_ref(q, k, v, do, rows, scale, cap, slopes)
        _attn_check(_attn_run(plan, mask, q, k, v, do, slopes), ref, f"scale {scale} cap {cap}")
