"""Attention at grids that fill the GPU: blocks of 128 rows or keys (from 512
blocks on), and blocks over keys that walk several query heads of theirs.
Many heads and few tokens, so that the float64 reference stays small."""

import math

import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log, rel_l2
from test_ops_gpu import ATTN_TOL, _attn_check, _attn_ref, _attn_run, _case
from test_ops_values_gpu import _formulas

pytestmark = pytest.mark.gpu


def _check(lens, pad, heads, kv, dim, kind, cap=0.0, bias=False, key_lens=None):
    q, k, v, do, mask, rows = _case(lens, pad, heads, kv, dim, kind, dim + heads, key_lens)
    slopes = 0.5 ** (torch.arange(heads) % 8 + 1.0) if bias else None
    plan = ops.Attn(len(rows), heads, dim, keys=len(k), kv_heads=kv, cap=cap)
    ref = _attn_ref(q, k, v, do, rows, 1 / math.sqrt(dim), cap, slopes)
    _attn_check(_attn_run(plan, mask, q, k, v, do, slopes), ref, f"{lens} {heads}/{kv} {dim}")


@pytest.mark.parametrize("dim", [40, 64, 88, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (5.0, False), (0.0, True), (50.0, True)])
def test_attn_blocks_of_128(dim, cap, bias):
    """Two blocks per head, the second with one row; ragged documents."""
    log(f"case attention 128-row blocks dim {dim} cap {cap} bias {bias}")
    _check([70, 1, 50], 8, 256, 256, dim, "causal", cap, bias)


@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("kind,lens,pad,heads", [
    ("doc", [193], 0, 256), ("prefix", [100, 93], 0, 256), ("causal", [257], 0, 176),
    ("doc", [1] * 60 + [69], 70, 256), ("causal", [128], 0, 512), ("doc", [], 130, 256),
])
def test_attn_blocks_of_128_masks(dim, kind, lens, pad, heads):
    log(f"case attention 128-row blocks dim {dim} {kind} {lens} pad {pad}")
    _check(lens, pad, heads, heads, dim, kind)


@pytest.mark.parametrize("dim", [64, 88, 128])
def test_attn_blocks_of_128_on_other_keys(dim):
    log(f"case attention 128-row blocks dim {dim} on other keys")
    _check([100, 80], 0, 256, 256, dim, "doc", key_lens=[33, 100])
    _check([20, 45], 0, 512, 512, dim, "causal", key_lens=[70, 3])


@pytest.mark.parametrize("dim,cap,bias", [(64, 0.0, False), (88, 20.0, True), (128, 0.0, True)])
def test_attn_key_blocks_that_walk_heads(dim, cap, bias):
    """1024 blocks of keys and more: each streams all the heads it serves."""
    log(f"case attention heads walked dim {dim}")
    _check([60, 69], 0, 1024, 512, dim, "causal", cap, bias)


@pytest.mark.parametrize("heads,kv,dim,cap", [
    (512, 64, 16, 0.0),   # 8 heads in parts of 2
    (511, 73, 16, 20.0),  # 7 heads in parts of 1, 2, 2 and 2
    (511, 73, 104, 0.0),
])
def test_attn_key_blocks_of_some_heads(heads, kv, dim, cap):
    """Key heads whose query heads fall to parts of several heads each."""
    log(f"case attention {heads} heads on {kv} in parts, dim {dim}")
    q, k, v, do, mask, rows = _case([64] * 25, 1, heads, kv, dim, "doc", dim)
    plan = ops.Attn(len(rows), heads, dim, kv_heads=kv, cap=cap)
    ref = _formulas(q, k, v, do, rows, 1 / math.sqrt(dim), cap)
    got = _attn_run(plan, mask, q, k, v, do)
    for n in ("o", "dq", "dk", "dv"):
        assert rel_l2(got[n], ref[n]) <= ATTN_TOL, n


@pytest.mark.parametrize("dim,bias", [(64, False), (64, True), (88, False), (88, True),
                                      (128, False), (128, True)])
def test_attn_blocks_of_128_under_a_large_cap(dim, bias):
    log(f"case attention 128-row blocks dim {dim} cap 1e4 bias {bias}")
    _check([70, 1, 50], 8, 256, 256, dim, "causal", 1e4, bias)
