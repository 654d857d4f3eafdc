"""Workspace sizes of attention over the whole range of shapes (no GPU): the
partial gradients of shared key heads stay within a bound, whatever the heads
and tokens.

The bound: fp32 partials of dk and dv for fewer than 7168 blocks of 128 keys,
7168 * 128 * head_dim * 4 * 2 bytes, beside D of every row.  (A key head's
blocks take parts of 1/3072 of what they would take together, rounded down to
whole heads: up to 6144 blocks, and one part more per key head, of which there
are fewer than 1024 blocks.)"""

import ctypes
import random

import pytest

from paper_2606_19163_amd import ops
from paper_2606_19163_amd import stage as S

from test_ops_host import built  # noqa: F401  (builds the library)


def _sizes(queries, keys, heads, kv, dim):
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    d = ops.AttnDesc(queries, keys, heads, kv, dim, 0.125, 0.0, S.BF16)
    assert ops.lib().pulse_attn_sizes(d, ctypes.byref(f), ctypes.byref(b)) == S.OK
    return f.value, b.value


def _bound(queries, heads, dim):
    return 7168 * 128 * dim * 8 + 4 * queries * heads + 4096


@pytest.mark.parametrize("queries,keys,heads,kv,dim", [
    (16000, 16000, 64, 8, 128), (65000, 65000, 32, 2, 128), (130000, 130000, 128, 1, 128),
    (130000, 131000, 1021, 1, 128), (1024, 131000, 1024, 1, 128), (5, 8000, 1024, 16, 64),
])
def test_backward_workspace_of_shared_heads(queries, keys, heads, kv, dim):
    assert _sizes(queries, keys, heads, kv, dim)[1] <= _bound(queries, heads, dim)


def test_backward_workspace_over_shapes():
    rng = random.Random(5)
    for _ in range(4000):
        kv = rng.choice((1, 1, 2, 3, 8, 40, 128))
        heads = kv * rng.randint(1, 1024 // kv)
        dim = 8 * rng.randint(1, 16)
        q, k = (int(2 ** rng.uniform(0, 20)) for _ in range(2))
        f, b = _sizes(q, k, heads, kv, dim)
        assert b <= _bound(q, heads, dim), (q, k, heads, kv, dim)
        # the forward's parts: at most one block of 64 rows per CU
        assert f <= 256 * 64 * (dim + 1) * 4 + 4096, (q, k, heads, kv, dim)
