"""Sparse steps at the borders of their kernels' forms, and values far apart."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn
from paper_2607_09207_b200 import workloads as W
from test_gpu_sparse import F8, chosen, close, host, i32, keys_of, pool, reference, run, run_select, select_case, summary_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nats", [6.0, 9.0, 12.0, 17.5, 19.0, 24.0])
@pytest.mark.parametrize("form", ["selected", "plain", "grouped", "scored"])
def test_many_small_weights_over_codes(nats, form):
    """A key that takes nearly all of the weight and has no V, over thousands of others."""
    bs, d, Hq, Hkv = 32, 128, 8, 2
    w = W.make_custom([20000, 20000, 300, 6000], Hq, Hkv, d, bs, seed=5, device="cuda:0")
    one, vs = torch.ones(2, device="cuda"), torch.full((2,), 0.03, device="cuda")
    k8, v8 = W.fp8_caches(w, one, vs)
    if form == "grouped":                                      # rows 0 and 1 share their first pages
        w.block_table[1, :300] = w.block_table[0, :300]
    k8.zero_()
    w.q.zero_()
    w.q[:, :, 0] = nats
    w.scale = 1.0
    table = w.block_table.cpu().numpy()
    for s, t in enumerate((700, 700, 5, 5999)):
        p, slot = int(table[s, t // bs]), t % bs
        k8[p, :, slot, 0] = 0x38                               # 1.0
        v8[p, :, :, slot] = 0
    k = k8.view(F8).double()
    v = v8.view(F8).double().transpose(2, 3) * vs.double().view(1, -1, 1, 1)
    P = w.block_table.shape[1]
    sel = np.broadcast_to(np.arange(P, dtype=np.int32), (4, Hkv, P))
    if form == "selected":
        got = [run(w, sel, hosted, fp8=(k8, v8, one, vs)) for hosted in (True, False)]
    else:
        out = torch.full_like(w.q, 7.0)
        args = (w.q, k8, v8, one, vs, w.block_table, w.context_lens, w.scale, out)
        if form == "plain":
            pdattn.decode_fp8(*args, pdattn.alloc_workspace(4, Hq, Hkv, d, bs))
        elif form == "scored":
            pdattn.decode_scored_fp8(*args, pdattn.alloc_workspace(4, Hq, Hkv, d, bs), pdattn.Score())
        else:
            pre = i32([150, 0])
            ws = pdattn.alloc_grouped_workspace(4, Hq, Hkv, d, bs)
            pdattn.decode_grouped_fp8(*args, ws, w.context_lens_host, 2, pre, pre.cpu().numpy())
        got = [out]
    want, size = reference(w, sel, k, v)
    for out in got:
        out = out.double().cpu().numpy()
        assert np.isfinite(out).all()
        # weights fp16, 2^-11 of each while they are normal, that is down to 2^-29 of the largest (20 nats); from there on off by at most half
        # of fp16's least step, 2^-25, beside a largest of 2^15: 2^-40 of that, 2^-40 e^nats of such a weight.  Scores and sums as in close()
        weights = max(2.0 ** -11, 2.0 ** -40 * math.exp(nats))
        tol = 2.0 ** -8 * abs(want) + (weights + 2.0 ** -12) * size + 1e-30
        assert (abs(out - want) <= tol).all(), (abs(out - want) / tol).max()


@pytest.mark.parametrize("fp8", [False, True])
def test_new_tokens_past_their_number_are_reported(fp8):
    """num_tokens below cu_tokens[S]: what lies past it is left out, and said so."""
    bs, d, Hkv = 16, 64, 2
    n = np.array([20, 40, 40])
    L = n + np.array([3, 0, 9])
    k, scale = pool(20, Hkv, bs, d, seed=3, fp8=fp8)
    table = np.arange(18).reshape(3, 6)
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    for num, served in ((100, 3), (101, 3), (99, 2), (60, 2), (59, 1), (1, 0)):
        s = pdattn.PageSummary.create(20, Hkv, d)
        s.exponents.fill_(99)
        pdattn.summarize_append(k, s, i32(table), i32(L), cu_tokens=i32([0, 20, 60, 100]), num_tokens=num, k_scale=scale, workspace=ws)
        assert pdattn.check(ws) == (pdattn.OK if served == 3 else pdattn.BAD_SEQUENCE), num
        filled = {int(table[r, b]) for r in range(served) for b in range((L[r] - n[r]) // bs, L[r] // bs)}
        assert set(np.flatnonzero((s.exponents.cpu().numpy() != 99).any(1)).tolist()) == filled, num


def test_pages_without_a_score_are_the_steps_to_report():
    """The choice looks at the table entries it scores; those it takes in any case go on as they are, and the step reports them."""
    w = W.make_custom([40 * 16, 5 * 16], 4, 2, 64, 16, device="cuda:0")
    s = pdattn.PageSummary.create(w.num_blocks, 2, 64)
    pdattn.summarize_pages(w.k_cache, s, i32(np.arange(w.num_blocks)))
    w.block_table[0, 0], w.block_table[0, 39], w.block_table[1, 2] = w.num_blocks + 3, -9, -1
    sel = torch.zeros(2, 2, 10, dtype=torch.int32, device="cuda")
    ws = pdattn.alloc_select_workspace(2, 2, w.block_table.shape[1])
    pdattn.select_pages(w.q, s, w.block_table, w.context_lens, sel, 16, ws, num_first=1, num_recent=1)
    assert pdattn.check(ws) == pdattn.OK
    assert (sel[0, :, 0] == 0).all() and (sel[0, :, 9] == 39).all() and (sel[1, :, :5].cpu() == torch.arange(5)).all()
    host_sel = sel.cpu().numpy()
    out = run(w, host_sel, hosted=False, expect=pdattn.BAD_PAGE_INDEX)
    left = host_sel.copy()
    left[0, :, [0, 9]] = -1
    left[1, :, 2] = -1
    close(out, *reference(w, left), 2.0 ** -15)


@pytest.mark.parametrize("S,pages", [(37, 2049), (74, 2049), (148, 2049), (148, 2048), (148, 2047)])
def test_selection_where_the_blocks_shares_change(S, pages):
    """As many (sequence, head) pairs as make a block score 512, 1024 and 2048 pages at a time; rows of 2047, 2048 and 2049 pages with a
    score among them, so that a row is one block's or two blocks' work, and a block's keys lie in its shared memory or not."""
    Hkv, first, recent = 4, 1, 2
    r = np.random.default_rng(S)
    rows = r.integers(1, 300, S)
    rows[:6] = [pages, 2047, 2048, min(pages, 2049), 513, 1025]
    rows[-2:] = [512, pages]
    rows = np.minimum(rows, pages) + first + recent
    L = rows * 16 - r.integers(0, 16, S)
    q, s, table = select_case(L, 8, Hkv, 64, 16, seed=S + pages, NB=5000, MB=pages + first + recent)
    got, st = run_select(q, s, table, L, 16, 40, first, recent)
    assert st == pdattn.OK
    some = np.r_[0:10, S - 4:S]
    assert (got[some] == chosen(q[some].double().cpu().numpy(), *host(q, s)[1:], table[some], L[some], 16, 40, first, recent)).all()


def test_long_rows_beside_more_units_than_the_workspace_numbers():
    """Above 2048 (sequence, head) pairs a block has a whole one, and its keys in memory where they are more than 2048."""
    L = np.random.default_rng(1).integers(1, 60 * 16, 700)
    L[[0, 1, 2, 350, 699]] = np.array([2200, 2052, 2051, 2199, 2050]) * 16
    q, s, table = select_case(L, 3, 3, 64, 16, seed=9, NB=4000)
    got, st = run_select(q, s, table, L, 16, 24, 1, 1)
    some = np.r_[0:5, 345:355, 690:700]
    assert st == pdattn.OK
    assert (got[some] == chosen(q[some].double().cpu().numpy(), *host(q, s)[1:], table[some], L[some], 16, 24, 1, 1)).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_draft_is_summarised_once_its_path_has_been_taken(fp8):
    """The accepted path overwrites slots of whole pages: their summaries follow it, by the accepted counts."""
    bs, d, Hkv, n, L = 16, 64, 2, np.array([16, 5]), np.array([36, 16])
    path = np.array([[0, 3, 4, 5, 7, 8, 9, 10, 12, 13, 14, 15], [1] + [-1] * 11])
    count = np.array([12, 1])                                       # 32 and 12 tokens stay
    k, scale = pool(8, Hkv, bs, d, seed=2, fp8=fp8)
    v = torch.zeros(8, Hkv, *((d, bs) if fp8 else (bs, d)), device="cuda", dtype=k.dtype)
    table, lens = i32([[4, 1, 6], [2, 3, 5]]), i32(L)
    s = pdattn.PageSummary.create(8, Hkv, d)
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    cu = i32(np.concatenate([[0], np.cumsum(n)]))
    pdattn.summarize_pages(k, s, i32([4, 1]), k_scale=scale)
    old = s.codes[1].clone()
    pdattn.tree_accept(k, v, table, lens, cu, i32(path), i32(count), workspace=ws)
    lens = i32(L - n + count)
    s.exponents.fill_(99)
    pdattn.summarize_append(k, s, table, lens, cu_tokens=i32([0, 12, 13]), num_tokens=13, k_scale=scale, workspace=ws)
    assert pdattn.check(ws) == pdattn.OK
    for h in range(Hkv):
        want = summary_of(keys_of(k, 1, h, scale))
        assert (s.codes[1, h].cpu().numpy() == want[0]).all() and int(s.exponents[1, h]) == want[1]
    assert not torch.equal(old, s.codes[1])
    assert (s.exponents[[0, 2, 3, 4, 5, 6, 7]] == 99).all()         # (page 2 of the second sequence is not whole any more)


@pytest.mark.parametrize("form", ["selected", "plain", "grouped", "scored"])
def test_v_scales_of_any_size(form):
    """A power of two as V's scale is the results' power of two, bit for bit."""
    bs, d, Hq, Hkv = 32, 128, 8, 2
    w = W.make_custom([20000, 20000, 300, 6000, 5, 64], Hq, Hkv, d, bs, seed=6, device="cuda:0")
    one = torch.ones(2, device="cuda")
    k8, v8 = W.fp8_caches(w, one, one * 0.03)
    w.block_table[1, :300] = w.block_table[0, :300]
    P = w.block_table.shape[1]
    sel = i32(np.broadcast_to(np.arange(P), (6, Hkv, P)))
    ws = pdattn.alloc_grouped_workspace(6, Hq, Hkv, d, bs)
    pre = i32([150, 0, 0])

    def call(vs):
        out = torch.full_like(w.q, 7.0)
        args = (w.q, k8, v8, one * 0.05, vs, w.block_table, w.context_lens)
        if form == "selected":
            pdattn.decode_selected_fp8(*args, sel, w.scale, out, ws)
        elif form == "plain":
            pdattn.decode_fp8(*args, w.scale, out, ws)
        elif form == "scored":
            pdattn.decode_scored_fp8(*args, w.scale, out, ws, pdattn.Score(window=5000))
        else:
            pdattn.decode_grouped_fp8(*args, w.scale, out, ws, w.context_lens_host, 2, pre, pre.cpu().numpy())
        assert pdattn.check(ws) == pdattn.OK
        return out.double()
    want = call(one)
    for k in (104, 60, -80):
        vs = torch.tensor([2.0 ** k, -(2.0 ** k)], device="cuda")
        out = call(vs)
        out[:, 4:] = -out[:, 4:]
        assert torch.equal(out, want * 2.0 ** k), k
