"""The plans of the products on a layer, without a GPU: each size of the table goes the way that it stands for, and there is no way that the table lacks."""
import math
import random

import pytest

import paper_1706_07191_amd as B
from tests.layer_sizes import PLANS, way_of


@pytest.mark.parametrize("name", PLANS)
def test_sizes_go_the_ways_that_they_stand_for(name):
    table, plan, contraction = PLANS[name]
    for way, size in table.items():
        p = plan(*size)
        assert way_of(p) == way, (size, p)
        k = contraction(*size)
        if way[0] == "rows":
            # of 64 numbers a chunk, four on their way; of 128 with 4-bit weights: two for each of eight waves and more
            assert k >= (2 * 8 * 128 if name == "linear" else 2 * 8 * 64 * (4 if way[1] == 1 else 2)) and k % 128 != 0
        else:
            _, _, _, tiles, large, _, parts, steps = p
            assert steps >= 9 and k - (parts - 1) * steps * 64 >= 9 * 64 - 63, (size, p)           # the last part too
            assert (large > 0) == (way[1] > 0) and (large == tiles or way[2] > 0)
            assert parts <= 16 and (parts - 1) * steps * 64 < k <= parts * steps * 64
            if name != "dX":
                assert k % 64 != 0
            else:
                assert size[2] % 64 != 0


@pytest.mark.parametrize("name", PLANS)
def test_no_size_goes_another_way(name):
    table, plan, _ = PLANS[name]
    rng = random.Random(7)
    for _ in range(40000):
        a, b, c = (int(math.exp(rng.uniform(0, math.log(most)))) for most in (20000, 40000, 40000))
        if rng.random() < 0.3:
            a = rng.randint(1, 64)
        assert way_of(plan(a, b, c)) in table, (a, b, c, plan(a, b, c))


@pytest.mark.parametrize("sizes", [(0, 5, 5), (5, 0, 5), (5, 5, 0), (-1, 5, 5), (1 << 31, 5, 5), (5, 5, 1 << 40)])
def test_refusals(sizes):
    for call in (lambda: B.brsvd_linear_e2m1_plan(*sizes), lambda: B.brsvd_linear_e2m1_plan(*sizes, True), lambda: B.brsvd_glu_plan(0, *sizes), lambda: B.brsvd_glu_plan(3, 5, 5, 5),
                 lambda: B.brsvd_glu_plan(-1, 5, 5, 5)):
        with pytest.raises(B.BrsvdError):
            call()
    assert B.lib().brsvd_linear_e2m1_plan(5, 5, 5, 0, None) == B.BRSVD_ERR_ARG and B.lib().brsvd_glu_plan(0, 5, 5, 5, None) == B.BRSVD_ERR_ARG
