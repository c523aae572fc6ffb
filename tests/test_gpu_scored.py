"""Single-token attention with modified scores and masks, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn
from paper_2607_09207_b200 import workloads as W

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def reference(w, cap=0.0, slopes=None, window=0, begin=None, k=None, v=None):
    """Output and sum of weight times |v|, in 64 bits; k, v: other caches than the workload's (already in 64 bits)."""
    S, Hq, d = w.q.shape
    G, bs = Hq // w.num_kv_heads, w.block_size
    k, v = (w.k_cache if k is None else k), (w.v_cache if v is None else v)
    out, size = torch.zeros(S, Hq, d, dtype=torch.double), torch.zeros(S, Hq, d, dtype=torch.double)
    for s in range(S):
        L = int(w.context_lens_host[s])
        lo = max(0, L - window if window else 0, int(begin[s]) if begin is not None else 0)
        if lo >= L:
            continue
        pg = w.block_table[s, :-(-L // bs)].long()
        kk, vv = (x[pg].transpose(0, 1).reshape(w.num_kv_heads, -1, d)[:, lo:L].double() for x in (k, v))
        x = torch.einsum("hgd,htd->hgt", w.q[s].double().view(-1, G, d), kk) * w.scale
        if cap:
            x = cap * torch.tanh(x / cap)
        if slopes is not None:
            x = x - slopes.double().view(-1, G, 1) * (L - 1 - torch.arange(lo, L, device=x.device))
        p = torch.softmax(x, -1)
        out[s] = torch.einsum("hgt,htd->hgd", p, vv).reshape(Hq, d).cpu()
        size[s] = torch.einsum("hgt,htd->hgd", p, vv.abs()).reshape(Hq, d).cpu()
    return out.numpy(), size.numpy()


def close(got, want, size, weights):
    # the result is rounded once (2^-8 of it); the weights carry `weights` relative to each, scores and sums are fp32 with
    # exponentials good to 2^-22 (below 2^-12 of sum p |v| for scores up to a few hundred)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    err, tol = abs(got - want), 2.0 ** -8 * abs(want) + (weights + 2.0 ** -12) * size + 1e-30
    assert (err <= tol).all(), (err / tol).max()


BF16_WEIGHTS = 2.0 ** -15        # two bf16 terms: 16 bits
F8_WEIGHTS = 2.0 ** -10          # fp16 weights (2^-11 each); q, bf16 of ordinary size, is exact in fp16


def run(w, host=True, slopes=None, window=0, begin=None, cap=0.0):
    ws = pdattn.alloc_workspace(w.num_seqs, w.num_q_heads, w.num_kv_heads, w.head_dim, w.block_size)
    out = torch.full_like(w.q, 7.0)
    sc = pdattn.Score(logit_cap=cap, bias_slopes=slopes, window=window,
                      key_begin=None if begin is None else torch.from_numpy(begin).cuda(), key_begin_host=begin if host else None)
    pdattn.decode_scored(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, out, ws, sc,
                         context_lens_host=w.context_lens_host if host else None)
    assert pdattn.check(ws) == pdattn.OK
    return out


def slopes_of(Hq):
    return (2.0 ** (-8.0 * (torch.arange(Hq, device="cuda") + 1) / Hq)).float()


LENS = [1, 2, 63, 64, 65, 0, 128, 700, 5000, 129, 1000, 17, 3]


@pytest.mark.parametrize("Hq,Hkv,d,bs", [(28, 4, 128, 16), (4, 1, 64, 16), (16, 1, 128, 32), (12, 1, 64, 64), (8, 8, 128, 64), (6, 2, 64, 32)])
@pytest.mark.parametrize("what", ["plain", "cap", "bias", "window", "document", "all"])
@pytest.mark.parametrize("host", [True, False])
def test_scores_and_masks(Hq, Hkv, d, bs, what, host):
    w = W.make_custom(LENS, Hq, Hkv, d, bs, seed=Hq, device="cuda:0")     # slots nobody owns hold NaN
    w.q.mul_(3.0)
    kw = {}
    if what in ("cap", "all"):
        kw["cap"] = 10.0
    if what in ("bias", "all"):
        kw["slopes"] = slopes_of(Hq)
    if what in ("window", "all"):
        kw["window"] = 100
    if what in ("document", "all"):
        kw["begin"] = np.array([0, 1, 62, 64, -5, 3, 128, 650, 4033, 128, 63, 17, 1], np.int32)   # some see nothing
    out = run(w, host=host, **kw)
    close(out, *reference(w, **kw), BF16_WEIGHTS)


@pytest.mark.parametrize("bs,d", [(16, 128), (32, 64), (64, 128)])
@pytest.mark.parametrize("host", [True, False])
def test_fp8_cache(bs, d, host):
    w = W.make_custom(LENS, 8, 2, d, bs, seed=3, device="cuda:0")
    ks, vs = torch.tensor([0.02, 0.03], device="cuda"), torch.tensor([0.03, 0.015], device="cuda")
    k8, v8 = W.fp8_caches(w, ks, vs)
    k = k8.view(F8).double() * ks.double().view(1, -1, 1, 1)
    v = v8.view(F8).double().transpose(2, 3) * vs.double().view(1, -1, 1, 1)
    for kw in ({}, dict(cap=8.0, slopes=slopes_of(8)), dict(window=90, begin=np.array([0, 1, 62, 64, -5, 3, 128, 650, 4033, 128, 63, 17, 1], np.int32))):
        begin = kw.get("begin")
        sc = pdattn.Score(logit_cap=kw.get("cap", 0.0), bias_slopes=kw.get("slopes"), window=kw.get("window", 0),
                          key_begin=None if begin is None else torch.from_numpy(begin).cuda(), key_begin_host=begin)
        ws = pdattn.alloc_workspace(w.num_seqs, 8, 2, d, bs)
        out = torch.full_like(w.q, 7.0)
        pdattn.decode_scored_fp8(w.q, k8, v8, ks, vs, w.block_table, w.context_lens, w.scale, out, ws, sc,
                                 context_lens_host=w.context_lens_host if host else None)
        assert pdattn.check(ws) == pdattn.OK
        close(out, *reference(w, k=k, v=v, **kw), F8_WEIGHTS)


def test_masked_places_may_hold_anything():
    w = W.make_custom([300, 64, 70], 8, 2, 128, 16, device="cuda:0")
    begin = np.array([150, 10, 66], np.int32)
    want = reference(w, begin=begin)
    bt = w.block_table.cpu().numpy()
    for s in range(3):
        for t in range(begin[s]):
            for x, bad in ((w.k_cache, math.inf), (w.v_cache, math.nan)):
                x[bt[s, t // 16], :, t % 16] = bad
    for host in (True, False):
        close(run(w, host=host, begin=begin), *want, BF16_WEIGHTS)


def test_nothing_asked_is_the_plain_step():
    w = W.make_config(2, device="cuda:0", num_seqs=40, len_div=4)
    a, b = run(w), torch.empty_like(w.q)
    ws = pdattn.alloc_workspace(w.num_seqs, w.num_q_heads, w.num_kv_heads, w.head_dim)
    pdattn.decode_ex(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, b, ws, context_lens_host=w.context_lens_host)
    assert torch.equal(a, b)


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_cut_units_in_every_merge_mode(mode):
    """Few long sequences: spans cut every unit, with leading tiles left out."""
    w = W.make_custom([9000, 20000, 64, 33000], 14, 2, 128, 16, seed=9, device="cuda:0")
    kw = dict(cap=20.0, begin=np.array([3000, 0, 63, 1], np.int32), window=25000)
    want = reference(w, **kw)
    pdattn.set_merge_mode(mode)
    try:
        a = run(w, **kw)
        assert torch.equal(run(w, **kw), a)
        close(a, *want, BF16_WEIGHTS)
        close(run(w, host=False, **kw), *want, BF16_WEIGHTS)
    finally:
        pdattn.set_merge_mode(-1)


def test_agrees_with_the_prompt_form():
    w = W.make_custom([5, 700, 130, 2000], 8, 2, 128, 16, device="cuda:0")
    sl = slopes_of(8)
    a, b = run(w, cap=15.0, slopes=sl, window=500), torch.empty_like(w.q)
    ws = pdattn.alloc_prefill_workspace(4, 4, 8, 2, 128)
    pdattn.prefill(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, torch.arange(5, dtype=torch.int32, device="cuda"), w.scale, b, ws,
                   score=pdattn.Score(logit_cap=15.0, bias_slopes=sl, window=500))
    _, size = reference(w, cap=15.0, slopes=sl, window=500)
    assert (abs(a.double() - b.double()).cpu().numpy() <= 2.0 ** -6 * size).all()


def test_captured_and_replayed():
    w = W.make_custom([300, 90, 500], 8, 2, 128, 16, device="cuda:0", poison=False)
    ws = pdattn.alloc_workspace(3, 8, 2, 128)
    out, begin = torch.empty_like(w.q), torch.zeros(3, dtype=torch.int32, device="cuda")
    sc = pdattn.Score(logit_cap=9.0, window=200, key_begin=begin)

    def call():
        pdattn.decode_scored(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, out, ws, sc)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    begin.copy_(torch.tensor([250, 89, 90]))
    w.context_lens.sub_(1)
    w.context_lens_host = w.context_lens_host - 1
    graph.replay()
    close(out, *reference(w, cap=9.0, window=200, begin=[250, 89, 90]), BF16_WEIGHTS)
    assert not out[1].any()


def test_wrapper_refuses_what_the_library_cannot_see():
    w = W.make_custom([30, 9], 8, 2, 64, 16, device="cuda:0")
    ws, out = pdattn.alloc_workspace(2, 8, 2, 64), torch.empty_like(w.q)
    args = [w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, out, ws]
    begin = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(pdattn.PdattnError):                               # host lengths, but no host copy of the first keys
        pdattn.decode_scored(*args, pdattn.Score(key_begin=begin), context_lens_host=w.context_lens_host)
    with pytest.raises(ValueError):
        pdattn.decode_scored(*args, pdattn.Score(key_begin=begin[:1]))
    with pytest.raises(ValueError):
        pdattn.decode_scored(*args, pdattn.Score(), context_lens_host=w.context_lens_host[:1])
    with pytest.raises(ValueError):
        pdattn.decode_scored(w.q[:1], *args[1:], pdattn.Score())
    with pytest.raises(TypeError):
        pdattn.Score(bias_slopes=torch.zeros(8, device="cuda", dtype=torch.double))


@pytest.mark.parametrize("cap", [1e-6, 0.5, 300.0, 1e4, 1e6])
def test_caps_far_from_the_scores(cap):
    """A cap far above the scores leaves them as they are to fp32 (tanh good to 2^-18 of small values: 2^-14 for scores
    up to 16), one far below makes them all alike."""
    w = W.make_custom([300, 64, 700], 8, 2, 128, 16, device="cuda:0")
    w.q.mul_(2.0)
    close(run(w, cap=cap), *reference(w, cap=cap), BF16_WEIGHTS)


@pytest.mark.parametrize("cap", [1e4, 3e4, 1e5, 1e6])
@pytest.mark.parametrize("X", [8192.0, -8192.0])
@pytest.mark.parametrize("fp8", [False, True])
def test_large_caps_keep_large_scores(cap, X, fp8):
    """Two keys whose logits agree: a score of X whose bias takes the capped score away, and a score of 0.  With v = 1 and -1 the
    output is tanh of half the logits' error.  Roundings of the first logit, in units of 2^-24 of it: tanh 8 (2^-21), its argument
    7, cap and product 3, slope 2, their sum 1; 24 are allowed for.  The weights: 2^-15, fp8 2^-11."""
    d = 128
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, kc, vc = (torch.zeros(s, device="cuda", dtype=BF16) for s in ((1, 2, d), (1, 1, 16, d), (1, 1, 16, d)))
    q[..., 3], kc[0, 0, 0, 3] = X / 64, 64.0
    vc[0, 0, 0], vc[0, 0, 1] = 1.0, -1.0
    out, ws = torch.empty_like(q), pdattn.alloc_workspace(1, 2, 1, d)
    sc = pdattn.Score(logit_cap=cap, bias_slopes=torch.full((2,), cap * math.tanh(X / cap), device="cuda"))
    if fp8:
        one = torch.ones(1, device="cuda")
        k8, v8 = kc.to(F8).view(torch.uint8), vc.to(F8).view(torch.uint8).transpose(2, 3).contiguous()
        pdattn.decode_scored_fp8(q, k8, v8, one, one, i32([[0]]), i32([2]), 1.0, out, ws, sc)
    else:
        pdattn.decode_scored(q, kc, vc, i32([[0]]), i32([2]), 1.0, out, ws, sc)
    assert pdattn.check(ws) == pdattn.OK
    # (the output is rounded once more, 2^-8 of a value below 0.01)
    assert float(out.float().abs().max()) <= (12 * 2.0 ** -24 * abs(X) + 2.0 ** -11) * (1 + 2.0 ** -8)


@pytest.mark.parametrize("L,key", [(600, 5), (600, 590), (9000, 40)])
def test_a_visible_infinity_of_vanishing_weight_is_never_lost(L, key):
    """A steep bias: the weight of a far key is 0 in 32 bits.  Its element is not finite all the same, the others are as ever."""
    w = W.make_custom([L, 70], 8, 2, 128, 16, device="cuda:0")
    slopes, page = torch.full((8,), 3.0, device="cuda"), int(w.block_table[0, key // 16])
    keep = w.v_cache[page, 1, key % 16, 9].clone()
    w.v_cache[page, 1, key % 16, 9] = math.inf
    for host in (True, False):
        out = run(w, host=host, slopes=slopes)
        w.v_cache[page, 1, key % 16, 9] = keep
        want, size = reference(w, slopes=slopes)
        w.v_cache[page, 1, key % 16, 9] = math.inf
        assert not out[0, 4:, 9].isfinite().any()
        out[0, 4:, 9] = 0.0
        want[0, 4:, 9] = 0.0
        close(out, want, size, BF16_WEIGHTS)
