"""The sizes of the linear layers' tile tests reach the kernels that they are listed under, and every
kernel that random sizes reach is listed; without a GPU, from the built library's own choice."""
import math
import random

import pytest

import linear_plan as lp


@pytest.mark.parametrize("table,kind,f32", [(lp.FORWARD_BF16, lp.FWD, False), (lp.FORWARD_F32, lp.FWD, True),
                                            (lp.DATA_GRADIENT, lp.DATA, False), (lp.WEIGHT_GRADIENT, lp.WEIGHT, False)])
def test_listed_sizes(table, kind, f32):
    for key, three in table.items():
        for i, s in enumerate(three):
            if s is None:
                assert key[0] == "64x64 any"
                continue
            tile, splits, sums = lp.plan(kind, *s, act=kind != lp.WEIGHT, f32=f32)
            assert (tile, splits > 1) + ((sums,) if kind == lp.WEIGHT else ()) == key, (key, s)
            m, k, n = s
            width, line = n if kind == lp.FWD else k, 32 if f32 or kind == lp.WEIGHT else 64  # of the result
            if i == 0:
                assert width % line == 0, (key, s)
            elif i == 1:
                assert width % 8 == 0 and width % line != 0, (key, s)
            else:
                assert k % 8 or n % 8, (key, s)


def test_few_rows():
    for m, k, n in lp.ROWS:
        assert lp.plan(lp.FWD, m, k, n, act=True) == ("rows", 1, False)
        assert lp.plan(lp.FWD, m, k, n, act=True, f32=True) == ("rows", 1, False)


def test_nothing_else_is_reached():
    rng = random.Random(11)
    size = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi))))  # noqa: E731
    for _ in range(20000):
        m, k, n, kind = size(1, 1e5), size(1, 16384), size(1, 16384), rng.randrange(3)
        f32 = kind == lp.FWD and rng.random() < 0.5
        tile, splits, sums = lp.plan(kind, m, k, n, act=rng.random() < 0.5, f32=f32)
        table = (lp.FORWARD_F32 if f32 else lp.FORWARD_BF16, lp.DATA_GRADIENT, lp.WEIGHT_GRADIENT)[kind]
        assert tile == "rows" or (tile, splits > 1) + ((sums,) if kind == lp.WEIGHT else ()) in table, (kind, m, k, n)
