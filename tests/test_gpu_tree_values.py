"""Attention for trees of drafted tokens where the inputs are not ordinary."""
import math

import numpy as np
import pytest
import torch

from test_gpu_tree import Case, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n", [4, 64])
@pytest.mark.parametrize("hist", [200, 9000])
def test_a_query_that_is_not_finite(fp8, n, hist):
    """Its row is NaN, whether its unit is cut (9000 keys) or not, in both forms; the other rows are as ever."""
    ns = np.array([n, 1, n - 1])
    c = Case(ns, ns + np.array([hist, 70, hist // 2]), 8, 2, 128, 16, seed=n, fp8=fp8)
    want, size = c.want()
    hit = [(0, 3), (n - 1, 6), (n + 1, 0), (2 * n - 1, 5)]
    for i, (row, head) in enumerate(hit):
        c.q[row, head, 5 * i] = (math.nan, math.inf, -math.inf, math.nan)[i]       # (an infinity: some scores are +inf)
    out = c.run()
    for row, head in hit:
        assert out[row, head].isnan().all(), (row, head)
        out[row, head], want[row, head], size[row, head] = 0, 0, 0
    close(out, want, size, fp8)


@pytest.mark.parametrize("n", [4, 64])
@pytest.mark.parametrize("hist", [200, 9000])
def test_scales_that_are_not_numbers(n, hist):
    ns = np.array([n, n])
    for what in ("scale", "k_scale", "v_scale"):
        c = Case(ns, ns + np.array([hist, 70]), 8, 2, 64, 32, seed=3, fp8=True)
        want, size = c.want()
        if what == "scale":
            c.scale = math.nan
            assert c.run().isnan().all()
            continue
        (c.ks if what == "k_scale" else c.vs)[1] = math.nan
        out = c.run()
        assert out[:, 4:].isnan().all()
        close(out[:, :4], want[:, :4], size[:, :4], True)
