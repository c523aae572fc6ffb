"""Attention for trees of drafted tokens where the inputs are not ordinary."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn
from test_gpu_tree import Case, close, i32

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


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n,hist", [(4, 700), (4, 9000), (64, 700), (64, 9000)])
@pytest.mark.parametrize("high", [0, 3, 6])
def test_values_that_are_not_finite_where_the_weight_vanishes(fp8, n, hist, high):
    """One key tile 500 above all others: an infinity or NaN of V in any other tile of the history still leaves its element not finite."""
    d, bs, heads = 64, 16, 4
    tiles = hist // 64
    for low in sorted({t for t in (0, 1, 2, 3, 4, 5, 6, 7, tiles - 1) if t != high}):
        c = Case([n], [n + hist], heads, 1, d, bs, seed=1, fp8=fp8)
        dead = (c.v.view(torch.float8_e4m3fn) if fp8 else c.v).float().isnan().any(2 if fp8 else 3)[:, 0]     # [page, slot]
        if fp8:
            c.ks.fill_(1.0)
        c.q.zero_()
        c.q[:, :, 0] = 8.0
        c.scale = 1.0
        c.k.zero_()
        key = np.arange(high * 64, high * 64 + 64)
        pages, slots = (torch.from_numpy(x).cuda() for x in (c.tab[0, key // bs].astype(np.int64), key % bs))
        c.k[pages, 0, slots, 0] = 0x6c if fp8 else 64.0                # 64 as a code is 0x68, 96 is 0x6c: 512 and 768 above the others
        want, size = c.want()
        bad = [(9, math.nan)] if fp8 else [(9, math.inf), (33, -math.inf), (50, math.nan)]
        for channel, x in bad:
            t = low * 64 + channel
            p, s = int(c.tab[0, t // bs]), t % bs
            assert not dead[p, s]
            if fp8:
                c.v[p, 0, channel, s] = 0x7f
            else:
                c.v[p, 0, s, channel] = x
        out = c.run()
        at = [ch for ch, _ in bad]
        assert not out[:, :, at].isfinite().any(), low
        out[:, :, at] = 0
        want[:, :, at], size[:, :, at] = 0, 0
        close(out, want, size, fp8)


def far_below(c, nats, sinks):
    """All keys score 0 but one per KV head, `nats` above, whose V is 0: what is left is the weights of the many."""
    c.ks.fill_(1.0)
    c.scale = 1.0
    c.k.zero_()
    c.q.zero_()
    c.q[:, :, 0] = nats
    for s, t in enumerate(sinks):
        p, slot = int(c.tab[s, t // c.bs]), t % c.bs
        c.k[p, :, slot, 0] = 0x38                          # 1.0
        c.v[p, :, :, slot] = 0


@pytest.mark.parametrize("nats", [6.0, 10.0, 14.0, 17.5, 18.5, 22.0])
@pytest.mark.parametrize("n", [4, 64])
@pytest.mark.parametrize("sink", ["first", "middle", "last"])
def test_many_small_weights_over_codes(nats, n, sink):
    """A key that takes nearly all of the weight and has no V, over thousands of others (the reference they are measured from)."""
    ns = np.array([n, 2, n])
    hist = np.array([30000, 400, 3000])
    c = Case(ns, ns + hist, 8, 2, 64, 32, seed=n, fp8=True)
    far_below(c, nats, {"first": [0] * 3, "middle": list(hist // 2), "last": list(hist - 1)}[sink])
    got = c.run().double().cpu().numpy()
    want, size = c.want()
    assert np.isfinite(got).all()
    # as in close(): weights fp16, 2^-11 of each while they are normal, that is down to 2^-24 of the largest (16.6 nats); from there on off by
    # at most half of fp16's least step, 2^-25, beside a largest of 2^10 or more: 2^-35 of that, 2^-35 e^nats of such a weight
    weights = max(2.0 ** -11, 2.0 ** -35 * math.exp(nats))
    tol = 2.0 ** -8 * abs(want) + (weights + 2.0 ** -12) * size + 1e-30
    err = abs(got - want)
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("n", [4, 64])
def test_scores_that_grow_and_are_large(n):
    """The maximum rises with every key tile, by little and by much, up to scores of some 10^6: no weight leaves fp16's range."""
    for step in (0.5, 2.0, 24.0):
        ns = np.array([n, n])
        c = Case(ns, ns + np.array([9000, 640]), 8, 2, 64, 32, seed=n, fp8=True)
        c.ks.fill_(1.0)
        c.k.zero_()
        c.q.zero_()
        # a key of tile t of the history scores q . k = 8 a + b/2 with t = 16 a + b (a < 16, b < 16), times the scale
        c.q[:, :, 0], c.q[:, :, 1] = 8.0, 0.5
        c.scale = 2.0 * step
        for s in range(2):
            for t in range(int(c.L[s]) // 64):
                key = np.arange(t * 64, t * 64 + 64)
                pages, slots = (torch.from_numpy(x).cuda() for x in (c.tab[s, key // 32].astype(np.int64), key % 32))
                for ch, x in ((0, t // 16), (1, t % 16)):
                    c.k[pages, :, slots, ch] = int(torch.tensor(float(x)).to(torch.float8_e4m3fn).view(torch.uint8))
        close(c.run(), *c.want(), True)
    c.q.mul_(512.0)                                          # one tile's keys, equal among themselves, take all
    close(c.run(), *c.want(), True)


@pytest.mark.parametrize("top", [8, 64])
@pytest.mark.parametrize("fp8", [False, True])
def test_ranges_of_tokens_that_are_none(top, fp8):
    """A sequence whose tokens are not all among the call's is left out, as before, and reported; the others are served."""
    n, L = np.array([5, 6, 3]), np.array([100, 260, 40])
    for cu, good in (([0, 5, 11, 15], (0, 1)), ([0, 5, 11, 1 << 30], (0, 1)), ([-1, 5, 11, 14], (1, 2)), ([0, 5, 4, 4], (0,)),
                     ([-(1 << 31), 5, 11, 14], (1, 2)), ([0, 5, 11, -(1 << 31)], (0, 1))):
        c = Case(n, L, 8, 2, 64, 16, fp8=fp8).upload()
        want, size = c.want()
        out = torch.full_like(c.q, 7.0)
        c.dev_cu = i32(cu)
        c.call(out, top)
        assert pdattn.check(c.ws) == pdattn.BAD_SEQUENCE, cu
        rows = np.concatenate([np.arange(int(c.cu[s]), int(c.cu[s + 1])) for s in good])
        close(out[rows], want[rows], size[rows], fp8)
        assert (out[np.setdiff1d(np.arange(14), rows)] == 7).all()
        out.fill_(7.0)                                       # (the workspace is as good as new)
        c.dev_cu = i32(c.cu)
        c.call(out, top)
        assert pdattn.check(c.ws) == pdattn.OK
        close(out, want, size, fp8)


@pytest.mark.parametrize("n", [4, 64])
@pytest.mark.parametrize("hist", [200, 9000])
def test_v_scales_of_any_size(n, hist):
    """A power of two as V's scale is the results' power of two, bit for bit, whether a unit is cut or not."""
    ns = np.array([n, 1, n])
    c = Case(ns, ns + np.array([hist, 3, hist // 3]), 8, 2, 128, 16, seed=7, fp8=True)
    c.vs.fill_(1.0)
    one = c.run()
    for k in (108, 60, -80):
        c.vs[0], c.vs[1] = 2.0 ** k, -(2.0 ** k)
        out = c.run().double()
        out[:, 4:] = -out[:, 4:]
        assert torch.equal(out, one.double() * 2.0 ** k), k
