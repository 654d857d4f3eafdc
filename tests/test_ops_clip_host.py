"""Which sets of gradients and outputs the clipping binding takes (no GPU)."""

import random

import pytest

from paper_2606_19163_amd import ops


@pytest.mark.parametrize("grads,outs", [
    ([], []),
    ([(0, 16), (16, 32)], [(0, 16), (16, 32)]),              # in place
    ([(0, 16), (8, 24)], [(100, 116), (116, 132)]),          # gradients are only read
    ([(0, 16), (0, 16)], [(100, 116), (116, 132)]),
    ([(0, 0), (0, 16)], [(4, 4), (0, 16)]),                  # an empty one is nowhere
    ([(64, 80), (0, 16)], [(64, 80), (32, 48)]),
])
def test_sets_that_are_taken(grads, outs):
    assert ops._clashes(grads, outs) is None


@pytest.mark.parametrize("grads,outs", [
    ([(0, 16), (0, 16)], [(0, 16), (0, 16)]),                # one gradient twice, in place
    ([(0, 16), (8, 24)], [(0, 16), (8, 24)]),
    ([(0, 16), (32, 48)], [(100, 116), (108, 124)]),         # outputs overlap
    ([(0, 16), (32, 48)], [(100, 116), (8, 24)]),            # another's gradient
    ([(0, 16)], [(4, 20)]),                                  # its own, moved
    ([(0, 64), (100, 104)], [(0, 64), (60, 64)]),
    ([(0, 200), (300, 304), (400, 404)], [(500, 700), (10, 14), (30, 34)]),
])
def test_sets_that_are_refused(grads, outs):
    assert ops._clashes(grads, outs) is not None


def test_against_every_pair():
    rng = random.Random(2)
    both = [0, 0]
    for _ in range(3000):
        n = rng.randint(1, 4)
        grads = [(b, b + rng.randint(0, 12)) for b in (rng.randint(0, 60) for _ in range(n))]
        outs = [g if rng.random() < 0.7 else (b, b + g[1] - g[0])
                for g, b in ((g, rng.randint(0, 90)) for g in grads)]

        def meet(x, y):
            return max(x[0], y[0]) < min(x[1], y[1])

        want = any(i != j and meet(outs[i], outs[j]) or
                   meet(outs[i], grads[j]) and not (i == j and outs[i] == grads[i])
                   for i in range(n) for j in range(n))
        assert (ops._clashes(grads, outs) is not None) == want, (grads, outs)
        both[want] += 1
    assert min(both) > 300
