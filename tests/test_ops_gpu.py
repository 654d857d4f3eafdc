"""The packed-sequence operators against plain float64 implementations on the
CPU, at the sizes, masks, strides and values where they can go wrong.

Tolerances.  u = 2^-8 is the unit roundoff of bf16 (half a spacing relative to
the value's binade).  A rounded bf16 output is off by at most u |value|; p and
ds are rounded to bf16 as operands, so a sum of products of them is off by at
most u times the sum of the absolute products, and D = rowsum(do o) sees o as
rounded.  In the relative L2 norm independent roundings of relative size
uniform in [-u, u] average to u / sqrt(3) = 2.3e-3 per rounding; an output
goes through at most three (p or ds, o in D, the output itself), so
sqrt(3) * 2.3e-3 = 4e-3 is expected where nothing cancels; 3 times that,
1.2e-2, is the bound.  fp32 turns: the angle's last rounding (2^-24 of half a
turn, 1.9e-7 rad), sin and cos (2^-23) and the products: below 1e-6 of the
pair's length."""

import math

import numpy as np
import pytest
import torch

from paper_2606_19163_amd import ops

from gpu_util import log, rel_l2

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
ATTN_TOL = 1.2e-2


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float32)


# ---- rotary positions ------------------------------------------------------------


def _rope_ref(x, pos, freq, dims, pairs, sign):
    x = x.double()
    axis = sum([[a] * (n // 2) for a, n in enumerate(dims)], [])
    ang = pos.double()[:, axis] * freq.double()
    c, s = torch.cos(ang)[:, None], sign * torch.sin(ang)[:, None]
    r = sum(dims)
    y = x.clone()
    i0 = range(0, r, 2) if pairs == "adjacent" else range(r // 2)
    i0 = torch.tensor(list(i0))
    i1 = i0 + 1 if pairs == "adjacent" else i0 + r // 2
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
@pytest.mark.parametrize("tokens,heads,dim,dims", [
    (1, 1, 8, [8]), (5, 3, 64, [16, 24, 24]), (7, 32, 88, [44, 44]), (33, 2, 128, [32, 40]),
    (258, 1, 256, [64, 64, 64, 64]), (3, 5, 40, [0, 40]), (1027, 13, 72, [24, 24, 24]),
])
def test_rope(dtype, pairs, tokens, heads, dim, dims):
    log(f"case rope {dtype} {pairs} {tokens}x{heads}x{dim} {dims}")
    g = _gen(tokens + dim)
    x = _randn(g, tokens, heads, dim).to(dtype)
    # positions below 0, between the grid points and far out: the angle is
    # reduced exactly, so a large one costs no accuracy
    pos = (_randn(g, tokens, len(dims)) * 50).round() / 2
    pos[0] = 65537.0
    freq = ops.rope_freqs(dims, device="cpu")
    plan = ops.Rope(heads, dim, dims, pairs=pairs, dtype=dtype)
    y = plan.forward(x.cuda(), pos.cuda(), freq.cuda())
    back = plan.backward(x.cuda(), pos.cuda(), freq.cuda())
    for got, sign in ((y, 1.0), (back, -1.0)):
        ref = _rope_ref(x, pos, freq, dims, pairs, sign)
        # per value: relative to its pair's largest possible length
        bound = (2.0 ** -8 if dtype == BF else 1e-6) * 1.01 * math.sqrt(2) * x.double().abs().max()
        assert (got.cpu().double() - ref).abs().max() <= bound
        assert rel_l2(got.cpu().double(), ref) <= (2.0 ** -8 if dtype == BF else 5e-7)


def test_rope_strided_in_place_and_alone():
    """The query and key heads inside a projection's output, turned in place:
    the value heads stay as they are, and a head-major output agrees."""
    g = _gen(3)
    t, h, d = 67, 4, 64
    qkv = _randn(g, t, 3 * h, d).to(BF).cuda()
    keep = qkv.clone()
    pos, freq = (_randn(g, t, 2) * 9).cuda(), ops.rope_freqs([32, 32])
    plan = ops.Rope(2 * h, d, [32, 32], pairs="halves")
    major = torch.empty(2 * h, t, d, dtype=BF, device="cuda").transpose(0, 1)
    plan.forward(qkv[:, :2 * h], pos, freq, out=major)
    plan.forward(qkv[:, :2 * h], pos, freq, out=qkv[:, :2 * h])
    assert torch.equal(qkv[:, 2 * h:], keep[:, 2 * h:])
    assert torch.equal(qkv[:, :2 * h], major)
    ref = _rope_ref(keep[:, :2 * h].cpu(), pos.cpu(), freq.cpu(), [32, 32], "halves", 1.0)
    assert rel_l2(major.cpu().double(), ref) <= 2.0 ** -8
    # a turn and its gradient undo one another (up to two roundings)
    x = _randn(g, t, 2 * h, d).cuda()
    f32 = ops.Rope(2 * h, d, [32, 32], pairs="halves", dtype=torch.float32)
    assert rel_l2(f32.backward(f32.forward(x, pos, freq), pos, freq).cpu(), x.cpu()) <= 1e-6
    assert f32.forward(x[:0], pos[:0], freq).shape == (0, 2 * h, d)


# ---- masks --------------------------------------------------------------------------


def _rows_ref(queries, keys, qo, ko, causal, prefix):
    rows = np.zeros((queries, 4), np.int64)
    rows[:, 3] = -1
    for d in range(len(qo) - 1):
        nq, nk = qo[d + 1] - qo[d], ko[d + 1] - ko[d]
        for r in range(nq):
            pos = ko[d] + r + nk - nq
            hi = ko[d + 1]
            if causal:
                hi = min(hi, max(pos + 1, ko[d] + (prefix[d] if prefix else 0)))
            lo = ko[d]
            if hi <= lo:
                lo = hi = 0
            rows[qo[d] + r] = (lo, hi, pos, d)
    return rows


def _tiles_ref(rows):
    out = []
    for a in range(0, len(rows), 64):
        t = rows[a:a + 64]
        live = t[t[:, 1] > t[:, 0]]
        lo, hi = (live[:, 0].min(), live[:, 1].max()) if len(live) else (0, 0)
        full = len(t) == 64
        out.append((lo, hi, t[:, 0].max(), t[:, 1].min() if full else 0))
    return np.array(out).reshape(-1, 4)


def _lens(rng, n, total, least=0):
    cut = np.sort(rng.integers(0, total - least * n + 1, n - 1))
    return (np.diff(np.concatenate([[0], cut, [total - least * n]])) + least).tolist()


def _off(lens):
    return [0] + np.cumsum(lens).tolist()


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", ["doc", "causal", "prefix"])
@pytest.mark.parametrize("queries,docs,pad", [
    (1, 1, 0), (63, 5, 3), (64, 1, 0), (65, 65, 0), (200, 150, 0), (1000, 7, 120), (777, 1, 777),
    (5000, 2000, 11),
])
def test_mask_of_documents(kind, queries, docs, pad):
    log(f"case mask {kind} {queries} rows {docs} documents {pad} padding")
    rng = np.random.default_rng(queries)
    qo = _off(_lens(rng, docs, queries - pad))
    causal = kind != "doc"
    prefix = [int(v) for v in rng.integers(0, 40, docs)] if kind == "prefix" else None
    m = ops.Mask(queries, docs=docs, causal=causal)
    rows = m.build(_dev(qo), prefix=None if prefix is None else _dev(prefix)).cpu().numpy()
    ref = _rows_ref(queries, queries, qo, qo, causal, prefix)
    assert np.array_equal(rows, ref)
    tiles = m.buffer[4 * queries:].cpu().numpy()[:4 * ((queries + 63) // 64)].reshape(-1, 4)
    assert np.array_equal(tiles, _tiles_ref(ref))


def test_mask_with_other_keys_and_empty_documents():
    qo, ko = [0, 3, 3, 10, 14], [0, 7, 9, 9, 11]
    for causal in (False, True):
        m = ops.Mask(16, keys=11, docs=4, causal=causal)
        rows = m.build(_dev(qo), key_offsets=_dev(ko)).cpu().numpy()
        assert np.array_equal(rows, _rows_ref(16, 11, qo, ko, causal, None))
    m = ops.Mask(5, docs=0)
    assert m.build(_dev([0])).cpu().tolist() == [[0, 0, 0, -1]] * 5
    assert ops.Mask(0, docs=1).build(_dev([0, 0])).shape == (0, 4)


def test_mask_clamps_what_memory_holds():
    """Offsets and rows that make no sense never leave the keys."""
    big = 2 ** 31 - 1
    for off in ([0, big, big, -big], [-5, 90, 10, 400], [7, 6, 5, 4], [-big, big, -big, big]):
        m = ops.Mask(100, keys=60, docs=3, causal=True)
        r = m.build(_dev(off), key_offsets=_dev(off), prefix=_dev([big, -big, 3])).cpu()
        assert (r[:, 0] >= 0).all() and (r[:, 1] <= 60).all() and (r[:, 1] >= r[:, 0]).all()
    m = ops.Mask(70, keys=60)
    m.rows.copy_(_dev([[-9, 1000, 3, 0], [50, 40, 2, 1]] * 35))
    r = m.from_rows(m.rows).cpu()
    assert r.tolist() == [[0, 60, 3, 0], [0, 0, 2, 1]] * 35


# ---- attention -------------------------------------------------------------------------


def _attn_ref(q, k, v, g, rows, scale, cap, slopes):
    """o, lse, dq, dk, dv in float64, head by head, from the formulas."""
    q, k, v, g = (x.double() for x in (q, k, v, g))
    tq, heads, d = q.shape
    tk, kv, _ = k.shape
    rep = heads // kv
    lo, hi, pos = (torch.as_tensor(rows[:, i]).long() for i in range(3))
    j = torch.arange(tk)
    see = (j >= lo[:, None]) & (j < hi[:, None])
    live = see.any(dim=1)
    o, dq = torch.zeros_like(q), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.full((heads, tq), -math.inf, dtype=torch.float64)
    for h in range(heads):
        n = h // rep
        kk, vv = k[:, n], v[:, n]
        # only what is attended is ever multiplied: the rest may hold NaN
        z = torch.full((tq, tk), -math.inf, dtype=torch.float64)
        raw = (q[:, h] @ kk.t()) * scale
        t = torch.tanh(raw / cap) if cap else torch.zeros_like(raw)
        raw = cap * t if cap else raw
        if slopes is not None:
            raw = raw - float(slopes[h]) * (pos[:, None] - j).abs().double()
        z[see] = raw[see]
        mx = z.amax(dim=1, keepdim=True)
        e = torch.where(see, torch.exp(z - mx), torch.zeros_like(z))
        s = e.sum(dim=1, keepdim=True)
        p = torch.where(live[:, None], e / s, torch.zeros_like(e))
        lse[h] = torch.where(live, (mx + torch.log(s))[:, 0], lse[h])
        dp = g[:, h] @ vv.t()
        o[:, h] = _see_mm(p, vv, see)
        D = torch.where(see, p * dp, torch.zeros_like(p)).sum(dim=1, keepdim=True)
        ds = torch.where(see, p * (dp - D) * (1 - t * t) * scale, torch.zeros_like(p))
        dq[:, h] = _see_mm(ds, kk, see)
        dk[:, n] += _see_mm(ds.t(), q[:, h], see.t())
        dv[:, n] += _see_mm(p.t(), g[:, h], see.t())
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv, alone_q=~live, alone_k=~see.any(dim=0))


def _see_mm(a, b, see):
    """sum over the seen positions only, also where b holds NaN or inf there."""
    bad = ~torch.isfinite(b).all(dim=1)
    c = a @ torch.where(bad[:, None], torch.zeros_like(b), b)
    for j in torch.nonzero(bad)[:, 0].tolist():
        c[see[:, j]] += a[see[:, j], j, None] * b[j]
    return c


def _attn_run(plan, mask, q, k, v, g, slopes=None):
    q, k, v, g = (x.cuda() for x in (q, k, v, g))
    sl = None if slopes is None else slopes.cuda()
    o, saved = plan.forward(q, k, v, mask, slopes=sl)
    dq, dk, dv = plan.backward(g, q, k, v, o, saved, mask, slopes=sl)
    torch.cuda.synchronize()
    return {n: x.cpu().double() for n, x in
            dict(o=o, lse=saved.lse, dq=dq, dk=dk, dv=dv).items()}


def _attn_check(got, ref, label):
    live = torch.isfinite(ref["lse"])
    assert torch.equal(torch.isfinite(got["lse"]), live), label
    assert (got["lse"][~live] == -math.inf).all()
    # lse: fp32 scores of |z| up to about 40 and their sum
    if live.any():
        assert (got["lse"][live] - ref["lse"][live]).abs().max() <= 2e-5, label
    errs = {n: rel_l2(got[n], ref[n]) if ref[n].abs().sum() > 0 else float(got[n].abs().sum())
            for n in ("o", "dq", "dk", "dv")}
    log(f"  {label}: " + ", ".join(f"{n} {e:.2e}" for n, e in errs.items()))
    for n, e in errs.items():
        assert e <= ATTN_TOL, (label, n, e)
    # rows and keys without a partner are exactly 0
    for n, alone in (("o", "alone_q"), ("dq", "alone_q"), ("dk", "alone_k"), ("dv", "alone_k")):
        assert (got[n][ref[alone]] == 0).all(), (label, n)


def _case(lens, pad, heads, kv, dim, kind, seed, key_lens=None):
    g = _gen(seed)
    tq = sum(lens) + pad
    tk = sum(key_lens) if key_lens else tq
    key_lens = key_lens[:len(lens)] if key_lens else None  # the rest is of no document
    q, do = (_randn(g, tq, heads, dim).to(BF) for _ in range(2))
    k, v = (_randn(g, tk, kv, dim).to(BF) for _ in range(2))
    prefix = [n // 3 for n in (key_lens or lens)]
    mask = ops.Mask(tq, keys=tk, docs=len(lens), causal=kind != "doc")
    ko = _off(key_lens) if key_lens else (_off(lens) if tk == tq else None)
    rows = mask.build(_dev(_off(lens)), key_offsets=_dev(ko),
                      prefix=_dev(prefix) if kind == "prefix" else None).cpu().numpy()
    return q, k, v, do, mask, rows


@pytest.mark.parametrize("dim", [8, 40, 64, 88, 96, 120, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (5.0, False), (0.0, True), (50.0, True)])
def test_attn_head_dims_caps_and_biases(dim, cap, bias):
    log(f"case attention dim {dim} cap {cap} bias {bias}")
    lens = [70, 1, 64, 130, 3]
    q, k, v, do, mask, rows = _case(lens, 9, 4, 2, dim, "doc", dim)
    slopes = torch.tensor([0.5, 0.05, 0.25, 0.0]) if bias else None
    plan = ops.Attn(len(rows), 4, dim, kv_heads=2, cap=cap)
    ref = _attn_ref(q, k, v, do, rows, 1 / math.sqrt(dim), cap, slopes)
    _attn_check(_attn_run(plan, mask, q, k, v, do, slopes), ref, f"dim {dim}")


@pytest.mark.parametrize("kind", ["doc", "causal", "prefix"])
@pytest.mark.parametrize("lens,pad", [
    ([1], 0), ([2], 3), ([63], 0), ([64], 0), ([65], 1), ([128], 0), ([129], 0), ([300], 0),
    ([1] * 70, 0), ([17, 0, 5, 111, 0, 64, 64, 1], 70), ([640], 100), ([], 66), ([257, 513], 1),
])
def test_attn_lengths_and_masks(kind, lens, pad):
    log(f"case attention lengths {lens} padding {pad} {kind}")
    q, k, v, do, mask, rows = _case(lens, pad, 3, 3, 64, kind, sum(lens))
    plan = ops.Attn(len(rows), 3, 64)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 0.0, None)
    _attn_check(_attn_run(plan, mask, q, k, v, do), ref, f"{kind} {lens}")


@pytest.mark.parametrize("heads,kv", [(1, 1), (6, 1), (8, 4), (5, 5)])
@pytest.mark.parametrize("lens,key_lens,kind", [
    ([200], [77], "doc"), ([100, 33], [1, 300], "doc"), ([1], [1000], "causal"),
    ([4], [515], "prefix"), ([90, 10], [30, 0], "causal"), ([1, 1, 1], [700, 5, 64], "doc"),
])
def test_attn_other_keys_and_shared_heads(heads, kv, lens, key_lens, kind):
    """Queries of another length than their keys: text tokens read by image
    tokens, new tokens after old ones, rows placed before their first key."""
    log(f"case attention {lens} over {key_lens} {kind} {heads}/{kv} heads")
    q, k, v, do, mask, rows = _case(lens, 0, heads, kv, 72, kind, heads, key_lens)
    plan = ops.Attn(sum(lens), heads, 72, keys=sum(key_lens), kv_heads=kv)
    ref = _attn_ref(q, k, v, do, rows, 1 / math.sqrt(72), 0.0, None)
    _attn_check(_attn_run(plan, mask, q, k, v, do), ref, f"{lens} over {key_lens}")


@pytest.mark.parametrize("lens,key_lens,kind,cap", [
    ([1], [5000], "causal", 0.0), ([3, 1], [2500, 2601], "doc", 9.0), ([70], [4096], "prefix", 0.0),
    ([2600], [33], "doc", 0.0), ([1500, 1200], [1, 130], "causal", 0.0), ([40], [3, ], "causal", 0.0),
    ([1] * 5, [1, 3000, 64, 0, 999], "doc", 0.0),
])
def test_attn_few_rows_over_a_long_axis(lens, key_lens, kind, cap):
    """Few blocks: the other side is split and the parts are joined."""
    log(f"case attention {lens} over {key_lens} {kind} in parts")
    for heads, kv, dim in ((2, 1, 64), (3, 3, 88), (1, 1, 128)):
        q, k, v, do, mask, rows = _case(lens, 2, heads, kv, dim, kind, dim, key_lens + [7])
        slopes = torch.tensor([0.01, 0.02, 0.0])[:heads] if cap else None
        plan = ops.Attn(len(rows), heads, dim, keys=sum(key_lens) + 7, kv_heads=kv, cap=cap)
        ref = _attn_ref(q, k, v, do, rows, 1 / math.sqrt(dim), cap, slopes)
        _attn_check(_attn_run(plan, mask, q, k, v, do, slopes), ref, f"{lens} over {key_lens}")


@pytest.mark.parametrize("lens,key_lens,heads,kv,kind", [
    ([1], [20011], 2, 1, "doc"),              # many parts for a row
    ([1, 0, 3, 1], [9000, 40, 0, 7011], 4, 4, "doc"),   # parts that see nothing of a document
    ([3000, 1, 2511], [90, 30, 81], 2, 1, "doc"),       # a document's rows fall to all parts
    ([1025], [1025], 2, 2, "causal"),
])
def test_attn_many_parts(lens, key_lens, heads, kv, kind):
    """The other side in up to 64 parts, for the keys every n-th tile of rows."""
    log(f"case attention {lens} over {key_lens}, {heads} heads on {kv}, {kind} in many parts")
    q, k, v, do, mask, rows = _case(lens, 3, heads, kv, 64, kind, 17, key_lens + [5])
    plan = ops.Attn(len(rows), heads, 64, keys=sum(key_lens) + 5, kv_heads=kv)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 0.0, None)
    _attn_check(_attn_run(plan, mask, q, k, v, do), ref, f"{lens} over {key_lens}")


def test_attn_nan_in_one_part():
    """A value that is not finite in a long axis stays with what attends it."""
    q, k, v, do, mask, rows = _case([40, 9], 1, 2, 1, 64, "causal", 21, [3000, 1500])
    plan = ops.Attn(50, 2, 64, keys=4500, kv_heads=1)
    v[2990, 0, 5] = math.inf  # of the rows placed there and later
    v[3100] = math.nan        # of the second document
    o, _ = plan.forward(q.cuda(), k.cuda(), v.cuda(), mask)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 0.0, None)["o"]
    o = o.cpu().double()
    assert torch.equal(torch.isnan(o), torch.isnan(ref))
    assert torch.equal(torch.isinf(o), torch.isinf(ref))
    ok = torch.isfinite(ref)
    assert rel_l2(o[ok], ref[ok]) <= ATTN_TOL


def test_attn_own_rows():
    """A window of keys around every row, rows in no order, some empty."""
    g = _gen(11)
    t, n = 333, 250
    q, do = (_randn(g, t, 2, 64).to(BF) for _ in range(2))
    k, v = (_randn(g, n, 2, 64).to(BF) for _ in range(2))
    mid = torch.randint(0, n, (t,), generator=g)
    rows = torch.stack([mid - 20, mid + torch.randint(-30, 60, (t,), generator=g), mid,
                        torch.zeros_like(mid)], dim=1).int()
    mask = ops.Mask(t, keys=n)
    rows = mask.from_rows(rows.cuda()).cpu().numpy()
    slopes = torch.tensor([0.1, 0.01])
    plan = ops.Attn(t, 2, 64, keys=n)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 0.0, slopes)
    _attn_check(_attn_run(plan, mask, q, k, v, do, slopes), ref, "windows")


@pytest.mark.parametrize("dim", [64, 88, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3.38e38])
def test_attn_values_in_masked_places(value, dim):
    """What a row does not attend does not reach it: the padding's rows hold
    only such values, and one document's are all of them."""
    log(f"case attention masked {value} dim {dim}")
    lens = [50, 40, 100]
    for kind in ("doc", "causal"):
        q, k, v, do, mask, rows = _case(lens, 30, 2, 1, dim, kind, 5)
        plan = ops.Attn(len(rows), 2, dim, kv_heads=1)
        clean = _attn_run(plan, mask, q, k, v, do)
        for x in (q, k, v, do):
            x[50:90] = value  # the second document
            x[190:] = value   # the padding
        got = _attn_run(plan, mask, q, k, v, do)
        for n in ("o", "dq", "dk", "dv"):
            keep = torch.cat([torch.arange(50), torch.arange(90, 190)])
            # bitwise: the same products, or sums of the same terms and zeros
            assert rel_l2(got[n][keep], clean[n][keep]) <= 1e-3, (kind, n)
            assert (got[n][190:] == 0).all(), (kind, n)


def test_attn_nan_of_a_later_key_stays_there():
    """Causal: a NaN in key and value 40 reaches the rows from 40 on only, in
    the channels it is in, and the gradients of what those rows touch."""
    q, k, v, do, mask, rows = _case([100], 0, 2, 2, 64, "causal", 6)
    v[40, 1, 7] = math.nan
    v[90, 0, 3] = math.inf
    plan = ops.Attn(100, 2, 64)
    o, _ = plan.forward(q.cuda(), k.cuda(), v.cuda(), mask)
    ref = _attn_ref(q, k, v, do, rows, 0.125, 0.0, None)["o"]
    o = o.cpu().double()
    assert torch.equal(torch.isnan(o), torch.isnan(ref))
    assert torch.equal(torch.isinf(o), torch.isinf(ref))
    ok = torch.isfinite(ref)
    assert rel_l2(o[ok], ref[ok]) <= ATTN_TOL


def test_attn_strides():
    """Heads inside a projection's output, head-major tensors, and a value
    that all tokens share (stride 0)."""
    g = _gen(12)
    t, h, d = 150, 4, 64
    qkv = _randn(g, t, h + 4, d).to(BF).cuda()
    q, k, v = qkv.split([h, 2, 2], dim=1)
    do = _randn(g, h, t, d).to(BF).cuda().transpose(0, 1)
    mask = ops.Mask(t, docs=2, causal=True)
    mask.build(_dev([0, 90, 140]))
    plan = ops.Attn(t, h, d, kv_heads=2)
    o, saved = plan.forward(q, k, v, mask)
    o2 = torch.empty(h, t, d, dtype=BF, device="cuda").transpose(0, 1)
    plan.forward(q.contiguous(), k.contiguous(), v.contiguous(), mask, out=o2)
    assert torch.equal(o, o2)
    a = plan.backward(do, q, k, v, o, saved, mask)
    dqkv = torch.full_like(qkv, 7.0)
    out = dqkv.split([h, 2, 2], dim=1)
    plan.backward(do.contiguous(), q, k, v, o2, saved, mask, out=out)
    for x, y in zip(a, out):
        assert torch.equal(x, y)
    one = v[:1].expand(t, 2, d)
    assert one.stride(0) == 0
    x, _ = plan.forward(q, k, one, mask)
    y, _ = plan.forward(q, k, one.contiguous(), mask)
    assert torch.equal(x, y)


def test_attn_gradient_against_differences():
    """<do, o(x + h dx) - o(x - h dx)> / 2h of the float64 formulas, in a
    direction of each input, against the kernels' gradients."""
    lens, heads, dim, cap = [33, 20], 2, 32, 4.0
    q, k, v, do, mask, rows = _case(lens, 5, heads, 1, dim, "prefix", 8)
    slopes = torch.tensor([0.2, 0.02])
    plan = ops.Attn(len(rows), heads, dim, kv_heads=1, cap=cap)
    got = _attn_run(plan, mask, q, k, v, do, slopes)
    g = _gen(9)
    h = 1e-5
    for n, x in (("dq", q), ("dk", k), ("dv", v)):
        # along the gradient itself, where nothing cancels
        dx = got[n] / got[n].norm()
        vals = []
        for s in (h, -h):
            args = {"dq": q.double(), "dk": k.double(), "dv": v.double()}
            args[n] = x.double() + s * dx
            o = _attn_ref(args["dq"], args["dk"], args["dv"], do, rows, 1 / math.sqrt(dim), cap,
                          slopes)["o"]
            vals.append(float((o * do.double()).sum()))
        fd = (vals[0] - vals[1]) / (2 * h)
        assert abs(fd - float((got[n] * dx).sum())) <= ATTN_TOL * abs(fd), n


def test_attn_long_cache_offsets():
    """Keys whose element offsets pass 2^31: a cache with a long stride per
    token of which this sequence is a part."""
    t, n, d, stride = 70, 600, 64, 1 << 22
    g = _gen(13)
    cache = torch.zeros((n - 1) * stride + 2 * d, dtype=BF, device="cuda")
    k, v = _randn(g, n, 1, d).to(BF), _randn(g, n, 1, d).to(BF)
    kc = cache.as_strided((n, 1, d), (stride, d, 1))
    vc = cache.as_strided((n, 1, d), (stride, d, 1), d)
    kc.copy_(k)
    vc.copy_(v)
    q = _randn(g, t, 1, d).to(BF)
    mask = ops.Mask(t, keys=n, docs=1, causal=True)
    rows = mask.build(_dev([0, t]), key_offsets=_dev([0, n])).cpu().numpy()
    plan = ops.Attn(t, 1, d, keys=n)
    o, _ = plan.forward(q.cuda(), kc, vc, mask)
    ref = _attn_ref(q, k, v, q, rows, 0.125, 0.0, None)["o"]
    assert rel_l2(o.cpu().double(), ref) <= ATTN_TOL


def test_attn_large_scores_and_scales():
    """Scores of hundreds, where exp of one alone overflows; a scale of 0."""
    q, k, v, do, mask, rows = _case([150], 0, 2, 2, 64, "causal", 14)
    for scale, mul in ((4.0, 4.0), (0.0, 1.0), (-0.125, 1.0)):
        plan = ops.Attn(150, 2, 64, scale=scale)
        qs = (q.float() * mul).to(BF)
        o, saved = plan.forward(qs.cuda(), k.cuda(), v.cuda(), mask)
        ref = _attn_ref(qs, k, v, do, rows, scale, 0.0, None)
        assert rel_l2(o.cpu().double(), ref["o"]) <= ATTN_TOL, scale
        assert rel_l2(saved.lse.cpu().double(), ref["lse"]) <= 1e-6, scale


def test_attn_streams_and_graph():
    """On a stream of its own, twice the same bits; captured and replayed with
    other inputs in the same place."""
    q, k, v, do, mask, rows = _case([200, 77], 3, 4, 2, 88, "doc", 15)
    plan = ops.Attn(len(rows), 4, 88, kv_heads=2)
    first = _attn_run(plan, mask, q, k, v, do)
    d = [x.cuda() for x in (q, k, v, do)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    o, saved = plan.forward(*d[:3], mask, stream=st)
    dq, dk, dv = plan.backward(d[3], *d[:3], o, saved, mask, stream=st)
    torch.cuda.synchronize()
    for n, x in dict(o=o, dq=dq, dk=dk, dv=dv).items():
        assert torch.equal(x.cpu().double(), first[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, saved = plan.forward(*d[:3], mask)
        dq, dk, dv = plan.backward(d[3], *d[:3], o, saved, mask)
    for seed in (1, 2, 3):
        g = _gen(seed)
        new = [_randn(g, *x.shape).to(BF) for x in d]
        for x, y in zip(d, new):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.cpu().double() for x in (o, dq, dk, dv)]
        want = _attn_run(plan, mask, *new)
        for x, n in zip(got, ("o", "dq", "dk", "dv")):
            assert torch.equal(x, want[n]), (seed, n)


# ---- gradient norm and clipping ----------------------------------------------------------


def _clip_ref(grads, max_norm, eps=1e-6):
    n = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    f = max_norm / (n + eps)
    return n, min(1.0, f)


@pytest.mark.parametrize("max_norm", [0.0, 1e-3, 1.0, 1e9])
@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [5, 8191, 8192, 8193, 1, 0, 70001], [300000]])
def test_clip(sizes, max_norm):
    log(f"case clip {sizes} {max_norm}")
    g = _gen(len(sizes))
    # views at odd element offsets of a shared buffer, both types
    flat = {t: _randn(g, sum(sizes) + len(sizes) + 8).to(t) for t in (torch.float32, BF)}
    views, at = [], 1
    for i, n in enumerate(sizes):
        views.append((BF if i % 2 else torch.float32, at, n))
        at += n + 1
    cpu = [flat[t][a:a + n] for t, a, n in views]
    dev = {t: x.cuda() for t, x in flat.items()}
    grads = [dev[t][a:a + n] for t, a, n in views]
    norm, f = _clip_ref(cpu, max_norm)
    outs = [torch.full((n + 3,), 5.0, dtype=t, device="cuda")[3:] for t, _, n in views]
    got = ops.GradClip(grads, outs=outs).run(max_norm)
    assert abs(float(got) - norm) <= 1e-6 * norm
    inplace = ops.GradClip(grads)
    assert float(inplace.run(max_norm)) == float(got)
    for i, (t, a, n) in enumerate(views):
        ref = cpu[i].double() * f
        # the factor is off by at most 4 fp32 roundings, the product is rounded once
        tol = (2.0 ** -8 if t == BF else 4e-7) * 1.01
        assert ((outs[i].cpu().double() - ref).abs() <= tol * ref.abs()).all()
        assert torch.equal(outs[i], grads[i])
    for t, x in dev.items():  # nothing between the views was touched
        live = torch.zeros(x.numel(), dtype=torch.bool)
        for u, a, n in views:
            if u == t:
                live[a:a + n] = True
        assert torch.equal(x.cpu()[~live], flat[t][~live])


def test_clip_range_and_nonfinite():
    """Squares beyond fp32, no tensors, and norms that are not finite."""
    x = torch.full((1000,), 1e30, device="cuda")
    n = ops.GradClip([x]).run(1.0)
    assert abs(float(n) / (1e30 * math.sqrt(1000)) - 1) <= 1e-6
    assert abs(float(x.double().norm()) - 1) <= 1e-6
    x = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(ops.GradClip([x]).run(1.0)) / (1e-30 * math.sqrt(1000)) - 1) <= 1e-6
    assert (x == 1e-30).all()
    assert float(ops.GradClip([]).run(1.0)) == 0.0
    y = torch.tensor([1.0, math.nan, 2.0], device="cuda")
    assert math.isnan(float(ops.GradClip([y]).run(1.0))) and torch.isnan(y).all()
    z = torch.tensor([1.0, math.inf, -2.0], device="cuda")
    assert float(ops.GradClip([z]).run(1.0)) == math.inf
    assert z[0] == 0 and torch.isnan(z[1]) and z[2] == 0


def test_clip_graph_replays():
    g = _gen(4)
    x = _randn(g, 50000).cuda()
    y = torch.empty_like(x)
    clip = ops.GradClip([x], outs=[y])
    clip.run(1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n = clip.run(1.0)
    for i in range(3):
        x.copy_(_randn(g, 50000) * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = (float(n), y.clone())
        assert float(clip.run(1.0)) == got[0] and torch.equal(y, got[1])
