"""Attention on NaN and infinities in attended places: o, lse and the
gradients are finite exactly where the float64 formulas are, and there they
are the formulas' values.

A key that a row attends reaches the row whatever tile both fall into, so the
documents here are shorter than a tile, cross tiles and hold a single token;
under a cap an infinite score is a finite one, +-cap."""

import math

import numpy as np
import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log
from test_ops_gpu import ATTN_TOL, _attn_run, _case

pytestmark = pytest.mark.gpu

LENS = [1, 40, 1, 3, 64, 70]


def _formulas(q, k, v, do, rows, scale, cap):
    """o, lse, dq, dk, dv in float64, over the keys that a row attends and no
    others: rows that attend the same keys are taken together."""
    q, k, v, do = (x.double().numpy() for x in (q, k, v, do))
    heads, rep = q.shape[1], q.shape[1] // k.shape[1]
    out = dict(o=np.zeros_like(q), lse=np.full((heads, len(q)), -np.inf), dq=np.zeros_like(q),
               dk=np.zeros_like(k), dv=np.zeros_like(v))
    spans, which = np.unique(rows[:, :2], axis=0, return_inverse=True)
    with np.errstate(all="ignore"):
        for s, (lo, hi) in enumerate(spans):
            i = np.flatnonzero(which.reshape(-1) == s)
            for h in range(heads if hi > lo else 0):
                n = h // rep
                qq, dd, kk, vv = q[i, h], do[i, h], k[lo:hi, n], v[lo:hi, n]
                z, t = qq @ kk.T * scale, 0.0
                if cap:
                    t = np.tanh(z / cap)
                    z = cap * t
                m = z.max(axis=1, keepdims=True)
                e = np.exp(z - m)
                p = e / e.sum(axis=1, keepdims=True)
                dp = dd @ vv.T
                ds = p * (dp - (p * dp).sum(axis=1, keepdims=True)) * (1 - t * t) * scale
                out["o"][i, h] = p @ vv
                out["lse"][h, i] = (m + np.log(e.sum(axis=1, keepdims=True)))[:, 0]
                out["dq"][i, h] = ds @ kk
                out["dk"][lo:hi, n] += ds.T @ qq
                out["dv"][lo:hi, n] += p.T @ dd
    return out


def _same_values(got, ref, label):
    """Finite where the reference is, and near it there."""
    for n in ("o", "lse", "dq", "dk", "dv"):
        r, g = ref[n], got[n].numpy()
        want, have = np.isfinite(r), np.isfinite(g)
        assert np.array_equal(have, want), (label, n, int((have != want).sum()))
        r, g = np.where(want, r, 0.0), np.where(want, g, 0.0)
        if n != "lse" and r.any():
            assert np.sqrt(((g - r) ** 2).sum()) <= ATTN_TOL * np.sqrt((r * r).sum()), (label, n)


def _values(x, name, value, cap, kind, dim, lens=LENS, heads=2, kv=1, key_lens=None):
    """The case with `value` in tensor `name`, rows or keys `x` of one head
    and channel 5 (and one whole row)."""
    q, k, v, do, mask, rows = _case(lens, 3, heads, kv, dim, kind, dim, key_lens)
    t = dict(q=q, k=k, v=v, do=do)[name]
    for i in x:
        t[i, 0, 5] = value
    plan = ops.Attn(len(rows), heads, dim, keys=len(k), kv_heads=kv, cap=cap)
    ref = _formulas(q, k, v, do, rows, 1 / math.sqrt(dim), cap)
    got = _attn_run(plan, mask, q, k, v, do)
    _same_values(got, ref, f"{name} {value} cap {cap} {kind} dim {dim}")


@pytest.mark.parametrize("dim", [64, 88, 128])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
def test_attn_values_reach_what_attends_them(name, value, cap, dim):
    log(f"case attention {name} {value} cap {cap} dim {dim}")
    for kind in ("doc", "causal"):
        # a one-token document, one inside a tile, one that crosses a tile
        for x in ([0], [20], [41], [43], [100], [44, 178]):
            _values(x, name, value, cap, kind, dim)


@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("value", [math.nan, -math.inf])
def test_attn_values_of_a_whole_document(name, value):
    """Every element of a document: its own rows and keys only."""
    q, k, v, do, mask, rows = _case(LENS, 3, 2, 2, 64, "doc", 7)
    dict(q=q, k=k, v=v, do=do)[name][1:41] = value
    plan = ops.Attn(len(rows), 2, 64)
    ref = _formulas(q, k, v, do, rows, 0.125, 0.0)
    _same_values(_attn_run(plan, mask, q, k, v, do), ref, f"{name} {value}")


@pytest.mark.parametrize("name,x", [("k", [700]), ("k", [2990]), ("v", [2990]), ("v", [3100]),
                                    ("q", [12]), ("do", [45])])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_attn_values_in_parts(name, x, value):
    """Few rows on a long axis, where the work is joined from parts."""
    log(f"case attention {name} {value} in parts")
    for cap in (0.0, 20.0):
        _values(x, name, value, cap, "causal", 64, [40, 9], 2, 1, [3000, 1500])


def test_attn_values_over_many_rows():
    """Many rows on few keys: the gradients of the keys come from parts."""
    for name, x in (("do", [1990]), ("q", [77]), ("k", [3]), ("v", [60])):
        _values(x, name, math.nan, 0.0, "doc", 64, [2600, 300], 1, 1, [33, 90])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("queries,keys", [(1, 6000), (40, 6000), (40, 500)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_attn_values_of_no_weight(value, queries, keys, dim):
    """A key that one far heavier leaves a weight of e^-200, 0 in fp32, is
    attended all the same."""
    log(f"case attention {value} of no weight, {queries} rows on {keys} keys, dim {dim}")
    for heavy, at in ((10, keys - 30), (keys - 30, 10), (keys - 30, keys // 2)):
        q, k, v, do, mask, rows = _case([queries], 2, 2, 1, dim, "doc", dim, [keys])
        q[:, :, 0] = 16.0
        k[:, :, 0] = 0.0
        k[heavy, :, 0] = 13.0 * math.sqrt(dim)
        v[at, 0, 5] = value
        plan = ops.Attn(len(rows), 2, dim, keys=keys, kv_heads=1)
        ref = _formulas(q, k, v, do, rows, 1 / math.sqrt(dim), 0.0)
        assert not np.isfinite(ref["o"][:queries, :, 5]).any()
        o, _ = plan.forward(q.cuda(), k.cuda(), v.cuda(), mask)
        assert np.array_equal(np.isfinite(o.float().cpu().numpy()), np.isfinite(ref["o"]))


def _time(f):
    """Best of three, in ms."""
    best = math.inf
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("name,rows", [("do", [9000]), ("do", None), ("v", [200]), ("v", None),
                                       ("k", [200]), ("k", None)])
def test_attn_values_do_not_stall_a_step(name, rows):
    """A diverged step (one NaN, or nothing but NaN) takes about as long as
    another: 3 times is allowed for what looks at the values once more."""
    t, h, d = 16384, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = {n: torch.randn(t, h, d, generator=gen, device="cuda").bfloat16()
         for n in ("q", "k", "v", "do")}
    mask = ops.Mask(t, docs=2, causal=True)
    mask.build(torch.tensor([0, 15000, 16384], dtype=torch.int32, device="cuda"))
    plan = ops.Attn(t, h, d)

    def step():
        o, saved = plan.forward(x["q"], x["k"], x["v"], mask)
        plan.backward(x["do"], x["q"], x["k"], x["v"], o, saved, mask)

    step()
    clean = _time(step)
    x[name][slice(None) if rows is None else rows] = math.nan
    odd = _time(step)
    log(f"  {name} {rows}: {clean:.2f} ms, with NaN {odd:.2f} ms")
    assert odd <= 3 * clean


@pytest.mark.parametrize("kind", ["doc", "causal"])
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_attn_values_at_a_scale_of_0(value, name, kind):
    """0 times infinity is no score of 0."""
    for x in ([0], [20], [100], [44, 178]):
        q, k, v, do, mask, rows = _case(LENS, 3, 2, 1, 64, kind, 64)
        for i in x:
            dict(q=q, k=k, v=v, do=do)[name][i, 0, 5] = value
        plan = ops.Attn(len(rows), 2, 64, kv_heads=1, scale=0.0)
        ref = _formulas(q, k, v, do, rows, 0.0, 0.0)
        _same_values(_attn_run(plan, mask, q, k, v, do), ref, f"{name} {value} {kind}")
