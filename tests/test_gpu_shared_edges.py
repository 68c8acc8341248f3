"""Edges of attention over shared pages: a scale of 0 times infinite and NaN elements of a query."""
import numpy as np
import pytest

from test_gpu_cache import BF, FP, f64, rand
from test_gpu_shared import INF, NAN, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,dtype", [(64, BF), (128, FP), (256, BF)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_scale_of_0_times_an_infinite_query(value, hd, dtype):
    """0 times an infinite or NaN element is NaN, whether the environment's keys are all shared or partly its own; other heads and
    environments are what they are without it."""
    H, K = 6, 2
    c = Case([(4, [0, 5, 33]), (5, [40, 0, 3, 100, 64])], K, hd, dtype, seed=hd)
    q = rand((c.n, H, hd), dtype, 1)
    want = f64(c.run(q, 0.0))
    for env in (0, 1, 2, 4):
        bad = q.clone()
        bad[env, 4, 9] = value
        got = f64(c.run(bad, 0.0))
        hit = np.zeros((c.n, H), bool)
        hit[env, 4] = True
        assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], want[~hit]), env
