"""Page summaries, the choice of pages by them and attention over the chosen pages, against their definitions."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn
from paper_2607_09207_b200 import workloads as W

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def exponent(a):
    """The smallest e in -40 .. 40 with a <= 127 * 2^e (Python integers and fractions: exact)."""
    e = -40
    while e < 40 and a > 127 * 2.0 ** e:
        e += 1
    return e


def summary_of(x):
    """Codes and exponent of one page-head x [slots, d] (float64)."""
    if not np.isfinite(x).all():
        return np.zeros((2, x.shape[1]), np.int8), 127
    lo, hi = x.min(0), x.max(0)
    e = exponent(max(abs(lo).max(), abs(hi).max()))
    return np.clip(np.stack([np.floor(lo / 2.0 ** e), np.ceil(hi / 2.0 ** e)]), -127, 127).astype(np.int8), e


def keys_of(k_cache, page, head, k_scale=None):
    x = k_cache[page, head]
    if k_cache.dtype == torch.uint8:
        x = x.view(F8).float() * k_scale[head]           # one fp32 product, by definition
    return x.double().cpu().numpy()


def pool(NB, Hkv, bs, d, seed=0, nhd=False, fp8=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fp8:
        k = (torch.randn(NB, Hkv, bs, d, device="cuda", generator=g) * 20).to(F8).view(torch.uint8)
        return k, torch.rand(Hkv, device="cuda", generator=g) * 0.05 + 0.01
    shape = (NB, bs, Hkv, d) if nhd else (NB, Hkv, bs, d)
    k = torch.randn(*shape, device="cuda", dtype=BF16, generator=g) * (2.0 ** torch.randint(-12, 12, (NB, 1, 1, 1), device="cuda", generator=g)).to(BF16)
    return (k.transpose(1, 2) if nhd else k), None


@pytest.mark.parametrize("bs,d,Hkv", [(16, 128, 4), (32, 64, 1), (64, 128, 9), (16, 64, 16), (64, 64, 2)])
@pytest.mark.parametrize("kind", ["bf16", "nhd", "fp8"])
def test_summaries(bs, d, Hkv, kind):
    NB = 23
    k, scale = pool(NB, Hkv, bs, d, seed=bs + d, nhd=kind == "nhd", fp8=kind == "fp8")
    k[3] = 0                                                     # zeros
    if kind != "fp8":
        k[4] = 1e-30                                             # far below the smallest exponent
        k[5, :, 1] = 3e38                                        # past the largest
        k[6, 0, bs - 1, d - 1] = math.nan
        k[7, Hkv - 1, 0, 0] = -math.inf
        k[8, :, :, 3] = -127.0                                   # the border of an exponent
        k[8, :, 0, 5] = 127.0
    else:
        k[6, 0, bs - 1, d - 1] = 0x7f
        k[7, Hkv - 1, 0, 0] = 0xff
    s = pdattn.PageSummary.create(NB, Hkv, d)
    s.codes.fill_(55)
    s.exponents.fill_(99)
    pages = np.array([3, 4, -1, 5, 6, 7, 8, 0, 22, 9, 9], np.int32)
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.summarize_pages(k, s, i32(pages), k_scale=scale, workspace=ws)
    assert pdattn.check(ws) == pdattn.OK
    codes, exps = s.codes.cpu().numpy(), s.exponents.cpu().numpy()
    for p in range(NB):
        for h in range(Hkv):
            want = summary_of(keys_of(k, p, h, scale)) if p in pages else (np.full((2, d), 55), 99)
            assert (codes[p, h] == want[0]).all() and exps[p, h] == want[1], (p, h)


@pytest.mark.parametrize("bs,d,fp8", [(16, 128, False), (32, 64, True), (64, 128, False)])
@pytest.mark.parametrize("one", [False, True])
def test_pages_filled_by_new_tokens(bs, d, fp8, one):
    """Chunks that end in, at and past a page's end, sequences without tokens, an empty one, a table row that is too short."""
    if one:
        L = np.array([1, bs - 1, bs, bs + 1, 3 * bs, 0, 5 * bs - 1, 4 * bs])
        n = np.ones(8, np.int64)
    else:
        L = np.array([5, bs, bs + 3, 4 * bs + 1, 3 * bs, 0, 2 * bs, 9 * bs, 7, 6 * bs])
        n = np.array([5, bs, 3, 2 * bs, 0, 0, 2 * bs + 4, 1, 7, bs + 1])
    S, MB, Hkv = len(L), 8, 3
    k, scale = pool(70, Hkv, bs, d, seed=3, fp8=fp8)
    table = np.random.default_rng(1).permutation(70)[:S * MB].reshape(S, MB) if S * MB <= 70 else np.random.default_rng(1).integers(0, 70, (S, MB))
    filled = set()
    late = False
    for s in range(S):
        for b in range(max(0, L[s] - n[s]) // bs, L[s] // bs):
            if b < MB:
                filled.add(int(table[s, b]))
            late |= b >= MB
    s = pdattn.PageSummary.create(70, Hkv, d)
    s.exponents.fill_(99)
    cu = np.concatenate([[0], np.cumsum(n)])
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.summarize_append(k, s, i32(table), i32(L), cu_tokens=None if one else i32(cu), num_tokens=int(cu[-1]), k_scale=scale, workspace=ws)
    assert pdattn.check(ws) == (pdattn.BAD_PAGE_INDEX if late else pdattn.OK)
    codes, exps = s.codes.cpu().numpy(), s.exponents.cpu().numpy()
    for p in range(70):
        for h in range(Hkv):
            want = summary_of(keys_of(k, p, h, scale)) if p in filled else (np.zeros((2, d)), 99)
            assert (codes[p, h] == want[0]).all() and exps[p, h] == want[1], (p, h)


@pytest.mark.parametrize("fp8", [False, True])
def test_the_least_keys_beside_the_largest(fp8):
    """A key below zero has a code below zero and one above zero a code above it, however small its share of the page's power of two."""
    d, bs = 128, 16
    if fp8:
        k = torch.zeros(2, 1, bs, d, dtype=torch.uint8, device="cuda")
        k[0, 0, 0, :4] = torch.tensor([0x7e, 0x81, 0x01, 0x80], dtype=torch.uint8, device="cuda")     # 448, -2^-9, 2^-9, -0
        scale = torch.tensor([2.0 ** 100], device="cuda")
        k[1, 0, :, :2] = torch.tensor([0x81, 0x01], dtype=torch.uint8, device="cuda")
        k[1, 0, :, 2] = 0x7e
    else:
        k = torch.zeros(2, 1, bs, d, dtype=BF16, device="cuda")
        k[0, 0, 0, :5] = torch.tensor([1e14, -1e-38, 1e-38, -0.0, 2.0 ** -133], dtype=torch.float64).to(BF16).cuda()
        k[1, 0, :, :3] = torch.tensor([2.0 ** 25, -(2.0 ** -133), 2.0 ** -133], dtype=torch.float64).to(BF16).cuda()
        scale = None
    s = pdattn.PageSummary.create(2, 1, d)
    pdattn.summarize_pages(k, s, i32([0, 1]), k_scale=scale)
    for p in range(2):
        want = summary_of(keys_of(k, p, 0, scale))
        assert (s.codes[p, 0].cpu().numpy() == want[0]).all() and int(s.exponents[p, 0]) == want[1]


def test_summary_of_a_page_that_is_none():
    k, _ = pool(5, 2, 16, 64)
    s = pdattn.PageSummary.create(5, 2, 64)
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.summarize_pages(k, s, i32([5, 1 << 30, 2]), workspace=ws)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX
    assert s.exponents[2].ne(0).any() and not s.codes[[0, 1, 3, 4]].any()


# ---------------------------------------------------------------------------------------------------------------
# Selection
# ---------------------------------------------------------------------------------------------------------------
def chosen(q, codes, exps, table, L, bs, K, first, recent):
    """The definition, page by page, in integers and float64 (exact: 21 bits times a power of two)."""
    S, Hq, d = q.shape
    Hkv = exps.shape[1]
    G, out = Hq // Hkv, np.full((S, Hkv, K), -1, np.int32)
    for s in range(S):
        P = min(-(-int(L[s]) // bs), table.shape[1])
        for h in range(Hkv):
            if P <= K:
                out[s, h, :P] = np.arange(P)
                continue
            score = np.full(P, -math.inf)
            ids = table[s, :P]
            ok = (ids >= 0) & (ids < len(exps))
            box, e_page = codes[np.where(ok, ids, 0), h].astype(np.int64), exps[np.where(ok, ids, 0), h].astype(np.float64)
            for x in q[s, h * G:h * G + G]:
                if not np.isfinite(x).all():
                    continue
                e = exponent(abs(x).max())
                c = np.clip(np.rint(x / 2.0 ** e), -127, 127).astype(np.int64)
                dot = np.maximum(c * box[:, 0], c * box[:, 1]).sum(-1)
                score = np.maximum(score, dot * 2.0 ** (e_page + e))
            score[e_page == 127] = math.inf
            rank = sorted(range(first, P - recent), key=lambda b: (not ok[b], -score[b], b))
            out[s, h] = sorted(list(range(first)) + rank[:K - first - recent] + list(range(P - recent, P)))
    return out


def select_case(L, Hq, Hkv, d, bs, seed=0, NB=None, MB=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = -(-np.asarray(L) // bs)
    MB = MB or max(1, int(pages.max()))
    NB = NB or int(pages.sum()) + 2
    r = np.random.default_rng(seed)
    table = np.full((len(L), MB), -1, np.int32)
    perm = r.permutation(NB) if NB >= pages.sum() else r.integers(0, NB, int(pages.sum()))
    at = 0
    for s in range(len(L)):
        n = min(pages[s], MB)
        table[s, :n] = perm[at:at + n]
        at += pages[s]
    q = torch.randn(len(L), Hq, d, device="cuda", dtype=BF16, generator=g)
    s = pdattn.PageSummary.create(NB, Hkv, d)
    mid = torch.randint(-90, 90, (NB, Hkv, 1, d), device="cuda", generator=g)
    wide = torch.randint(0, 37, (NB, Hkv, 1, d), device="cuda", generator=g)
    s.codes.copy_(torch.cat((mid - wide, mid + wide), 2))
    s.exponents.copy_(torch.randint(-7, -3, (NB, Hkv), device="cuda", generator=g))
    return q, s, table


def run_select(q, s, table, L, bs, K, first, recent, ws=None):
    S, Hkv = len(L), s.exponents.shape[1]
    out = torch.full((S, Hkv, K), 77, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = pdattn.alloc_select_workspace(S, Hkv, table.shape[1])
    pdattn.select_pages(q, s, i32(table), i32(L), out, bs, ws, num_first=first, num_recent=recent)
    return out.cpu().numpy(), pdattn.check(ws)


def host(q, s):
    return q.double().cpu().numpy(), s.codes.cpu().numpy(), s.exponents.cpu().numpy()


@pytest.mark.parametrize("Hq,Hkv,d,bs", [(28, 4, 128, 16), (4, 1, 64, 16), (16, 1, 128, 32), (12, 1, 64, 64), (3, 3, 128, 64)])
@pytest.mark.parametrize("K,first,recent", [(1, 0, 1), (8, 1, 2), (9, 0, 1), (33, 4, 1), (3, 1, 2)])
def test_selection(Hq, Hkv, d, bs, K, first, recent):
    L = np.array([0, 1, bs, 8 * bs, 8 * bs + 1, 33 * bs, 34 * bs, 40 * bs - 3, 600 * bs + 5, 1100 * bs, 517 * bs])
    q, s, table = select_case(L, Hq, Hkv, d, bs, seed=K)
    got, st = run_select(q, s, table, L, bs, K, first, recent)
    assert st == pdattn.OK
    assert (got == chosen(*host(q, s), table, L, bs, K, first, recent)).all()


@pytest.mark.parametrize("pages,K", [(2040, 512), (2060, 100), (8200, 7), (8300, 4000), (20000, 300)])
def test_selection_of_long_contexts(pages, K):
    """Keys held eight and 32 to a thread, and read again in every round."""
    L = np.array([pages * 16 - 5, 100])
    q, s, table = select_case(L, 8, 2, 64, 16, seed=pages, NB=3000)
    got, st = run_select(q, s, table, L, 16, K, 2, 3)
    assert st == pdattn.OK and (got == chosen(*host(q, s), table, L, 16, K, 2, 3)).all()


def test_equal_scores_go_to_the_first_pages():
    L = np.array([900 * 16, 2500 * 16])
    q, s, table = select_case(L, 8, 2, 128, 16, seed=5)
    s.codes.copy_(s.codes[:1].expand_as(s.codes).clone())
    s.exponents.fill_(-5)
    got, _ = run_select(q, s, table, L, 16, 40, 1, 2)
    for r in range(2):
        n = L[r] // 16
        assert (got[r] == np.concatenate([np.arange(38), [n - 2, n - 1]])).all()
    s.exponents[table[1, 1500:1510]] = 3                       # (positive scores grow with the exponent: bounds of q . k over a box)
    got, _ = run_select(q, s, table, L, 16, 40, 1, 2)
    assert (got == chosen(*host(q, s), table, L, 16, 40, 1, 2)).all()


def test_values_that_are_not_finite():
    L = np.array([300 * 16, 300 * 16, 300 * 16])
    q, s, table = select_case(L, 8, 2, 64, 16, seed=6)
    s.exponents[table[0, 200]] = 127                           # keys that are not finite: always in
    s.codes[table[0, 200]] = 0
    q[1, 2, 5] = math.nan                                      # one head of a group takes no part
    q[1, 3, 0] = math.inf
    q[2, :4] = -math.inf                                       # no head is left: the first pages
    q[2, 5] = 3e38                                             # codes saturate
    q[2, 6] = 1e-30
    q[2, 7] = 0
    got, st = run_select(q, s, table, L, 16, 20, 0, 1)
    assert st == pdattn.OK and (got == chosen(*host(q, s), table, L, 16, 20, 0, 1)).all()
    assert (got[0] == 200).any(-1).all() and (got[2, 0] == np.r_[0:19, 299]).all()


def test_bad_pages_and_short_rows_are_reported():
    L = np.array([100 * 16, 90 * 16])
    q, s, table = select_case(L, 4, 2, 64, 16, seed=7, MB=90)
    got, st = run_select(q, s, table, L, 16, 10, 1, 1)
    assert st == pdattn.BAD_PAGE_INDEX and (got == chosen(*host(q, s), table, L, 16, 10, 1, 1)).all()
    L[0] = 90 * 16
    table[1, 30], table[1, 31] = -7, 1 << 30
    ws = pdattn.alloc_select_workspace(2, 2, 90)
    got, st = run_select(q, s, table, L, 16, 10, 1, 1, ws)
    assert st == pdattn.BAD_PAGE_INDEX and (got == chosen(*host(q, s), table, L, 16, 10, 1, 1)).all()
    table[1, 30:32] = table[1, :2]
    got, st = run_select(q, s, table, L, 16, 10, 1, 1, ws)
    assert st == pdattn.OK and (got == chosen(*host(q, s), table, L, 16, 10, 1, 1)).all()


def test_more_units_than_the_workspace_numbers():
    """Above 2048 (sequence, head) pairs a block scores a whole one."""
    L = np.random.default_rng(0).integers(1, 700 * 16, 700)
    L[:3] = 700 * 16
    q, s, table = select_case(L, 3, 3, 64, 16, seed=8, NB=4000)
    got, st = run_select(q, s, table, L, 16, 24, 1, 1)
    some = np.r_[0:8, 690:700]
    assert st == pdattn.OK
    assert (got[some] == chosen(q[some].double().cpu().numpy(), *host(q, s)[1:], table[some], L[some], 16, 24, 1, 1)).all()


# ---------------------------------------------------------------------------------------------------------------
# Attention over chosen pages
# ---------------------------------------------------------------------------------------------------------------
def reference(w, sel, k=None, v=None):
    """Output and sum of weight times |v|, in 64 bits."""
    S, Hq, d = w.q.shape
    Hkv, bs = w.num_kv_heads, w.block_size
    G = Hq // Hkv
    k, v = (w.k_cache if k is None else k), (w.v_cache if v is None else v)
    table = w.block_table.cpu().numpy()
    out, size = np.zeros((S, Hq, d)), np.zeros((S, Hq, d))
    for s in range(S):
        L = int(w.context_lens_host[s])
        P = -(-L // bs)
        for h in range(Hkv):
            b = [int(x) for x in sel[s, h, :min(sel.shape[2], P)] if 0 <= x < P]
            at = [(int(table[s, x]), t) for x in b for t in range(min(bs, L - x * bs))]
            if not at:
                continue
            pg, sl = (torch.tensor(x, device=w.q.device) for x in zip(*at))
            kk, vv = k[pg, h, sl].double(), v[pg, h, sl].double()
            p = torch.softmax(w.q[s, h * G:h * G + G].double() @ kk.T * w.scale, -1)
            out[s, h * G:h * G + G] = (p @ vv).cpu().numpy()
            size[s, h * G:h * G + G] = (p @ vv.abs()).cpu().numpy()
    return out, size


def close(got, want, size, weights):
    # the result is rounded once (2^-8 of it); the weights carry `weights` relative to each, scores and sums are fp32 with
    # exponentials good to 2^-22 (below 2^-12 of sum p |v| for scores up to a few hundred)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    err, tol = abs(got - want), 2.0 ** -8 * abs(want) + (weights + 2.0 ** -12) * size + 1e-30
    assert (err <= tol).all(), (err / tol).max()


BF16_WEIGHTS = 2.0 ** -15        # two bf16 terms: 16 bits
F8_WEIGHTS = 2.0 ** -10          # fp16 weights (2^-11 each); q, bf16 of ordinary size, is exact in fp16


def run(w, sel, hosted=True, fp8=None, expect=pdattn.OK):
    ws = pdattn.alloc_workspace(w.num_seqs, w.num_q_heads, w.num_kv_heads, w.head_dim, w.block_size)
    out = torch.full_like(w.q, 7.0)
    lens = w.context_lens_host if hosted else None
    if fp8 is None:
        pdattn.decode_selected(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, i32(sel), w.scale, out, ws, context_lens_host=lens)
    else:
        pdattn.decode_selected_fp8(w.q, *fp8, w.block_table, w.context_lens, i32(sel), w.scale, out, ws, context_lens_host=lens)
    assert pdattn.check(ws) == expect
    return out


LENS = [1, 2, 63, 64, 65, 0, 128, 700, 5000, 129, 1000, 17, 3]


def lists(w, K, seed=0, order="ascending"):
    """Distinct pages of every sequence, the last one among them."""
    r = np.random.default_rng(seed)
    sel = np.full((w.num_seqs, w.num_kv_heads, K), -1, np.int32)
    for s in range(w.num_seqs):
        P = -(-int(w.context_lens_host[s]) // w.block_size)
        for h in range(w.num_kv_heads):
            n = min(P, K)
            if n:
                b = np.concatenate([r.permutation(P - 1)[:n - 1], [P - 1]])
                sel[s, h, :n] = np.sort(b) if order == "ascending" else r.permutation(b)
    return sel


@pytest.mark.parametrize("Hq,Hkv,d,bs", [(28, 4, 128, 16), (4, 1, 64, 16), (16, 1, 128, 32), (12, 1, 64, 64), (8, 8, 128, 64), (6, 2, 64, 32)])
@pytest.mark.parametrize("K", [1, 2, 5, 37, 500])
@pytest.mark.parametrize("hosted", [True, False])
def test_chosen_pages(Hq, Hkv, d, bs, K, hosted):
    w = W.make_custom(LENS, Hq, Hkv, d, bs, seed=Hq, device="cuda:0")     # slots nobody owns hold NaN
    for order in ("ascending", "any"):
        sel = lists(w, K, order=order)
        close(run(w, sel, hosted), *reference(w, sel), BF16_WEIGHTS)


@pytest.mark.parametrize("bs,d", [(16, 128), (32, 64), (64, 128), (16, 64)])
@pytest.mark.parametrize("K", [1, 3, 30])
def test_fp8_cache(bs, d, K):
    w = W.make_custom(LENS, 8, 2, d, bs, seed=3, device="cuda:0")
    ks, vs = torch.tensor([0.02, 0.03], device="cuda"), torch.tensor([0.03, 0.015], device="cuda")
    k8, v8 = W.fp8_caches(w, ks, vs)
    k = k8.view(F8).double() * ks.double().view(1, -1, 1, 1)
    v = v8.view(F8).double().transpose(2, 3) * vs.double().view(1, -1, 1, 1)
    for order in ("ascending", "any"):
        sel = lists(w, K, order=order)
        for hosted in (True, False):
            close(run(w, sel, hosted, fp8=(k8, v8, ks, vs)), *reference(w, sel, k, v), F8_WEIGHTS)


def test_all_pages_are_the_plain_step():
    w = W.make_config(2, device="cuda:0", num_seqs=40, len_div=4)
    P = w.block_table.shape[1]
    sel = np.broadcast_to(np.arange(P, dtype=np.int32), (40, w.num_kv_heads, P))
    b = torch.empty_like(w.q)
    ws = pdattn.alloc_workspace(w.num_seqs, w.num_q_heads, w.num_kv_heads, w.head_dim)
    pdattn.decode_ex(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, b, ws, context_lens_host=w.context_lens_host)
    assert torch.equal(run(w, sel), b)


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_cut_units_in_every_merge_mode(mode):
    w = W.make_custom([9000, 20000, 64, 33000], 14, 2, 128, 16, seed=9, device="cuda:0")
    sel = lists(w, 700)
    pdattn.set_merge_mode(mode)
    try:
        a = run(w, sel)
        assert torch.equal(run(w, sel), a)
        close(a, *reference(w, sel), BF16_WEIGHTS)
        close(run(w, sel, hosted=False), *reference(w, sel), BF16_WEIGHTS)
    finally:
        pdattn.set_merge_mode(-1)


@pytest.mark.parametrize("fp8", [False, True])
def test_gaps_repeats_and_what_is_not_chosen(fp8):
    """Entries below zero anywhere, a page named twice (the partial one too), nothing chosen at all; pages that are not chosen hold NaN."""
    w = W.make_custom([300, 70, 200, 90, 16 * 40], 8, 2, 128, 16, device="cuda:0")
    sel = np.full((5, 2, 12), -1, np.int32)
    sel[0, 0, [1, 5, 11]] = 18, 3, 0
    sel[0, 1, :5] = 7, 18, 7, 18, 2
    sel[1, :, :3] = 4                                          # the partial page three times in one tile
    sel[2, 0, 3] = 12
    sel[4, 0] = np.arange(12) * 3
    sel[4, 1, ::2] = 39
    used = {(int(w.block_table[s, b]), h) for s in range(5) for h in range(2)
            for b in sel[s, h, :min(12, -(-int(w.context_lens_host[s]) // 16))] if b >= 0}
    for p in range(w.num_blocks):
        for h in range(2):
            if (p, h) not in used:
                w.k_cache[p, h], w.v_cache[p, h] = math.nan, math.nan
    if fp8:
        one = torch.full((2,), 0.02, device="cuda")
        k8, v8 = W.fp8_caches(w, one, one)
        k, v = k8.view(F8).double() * 0.02, v8.view(F8).double().transpose(2, 3) * 0.02
        # (0.02 is a float: the product's scale differs from the double by 2^-25 of it)
        kw, args, tol = dict(fp8=(k8, v8, one, one)), (k, v), F8_WEIGHTS
    else:
        kw, args, tol = {}, (), BF16_WEIGHTS
    for hosted in (True, False):
        out = run(w, sel, hosted, **kw)
        close(out, *reference(w, sel, *args), tol)
        assert not out[3].any() and not out[2, 4:].any()


def test_pages_that_the_sequence_does_not_have():
    w = W.make_custom([300, 70, 500], 8, 2, 64, 16, device="cuda:0")
    sel = lists(w, 8)
    sel[0, 1, 3] = 19                                          # 300 tokens: pages 0 .. 18
    out = run(w, sel, expect=pdattn.BAD_PAGE_INDEX)
    close(out, *reference(w, sel), BF16_WEIGHTS)
    w.block_table[2, int(sel[2, 0, 2])] = w.num_blocks + 5     # a table entry that is no page
    bad = sel.copy()
    for h in range(2):
        bad[2, h][bad[2, h] == sel[2, 0, 2]] = -1
    out = run(w, sel, expect=pdattn.BAD_PAGE_INDEX)
    close(out, *reference(w, bad), BF16_WEIGHTS)


def test_a_step_captured_and_replayed():
    """Append's lengths, summaries, choice and attention in one graph; another step's inputs on replay."""
    bs, K = 16, 9
    w = W.make_custom([300, 90, 500], 8, 2, 128, bs, device="cuda:0", poison=False)
    s = pdattn.PageSummary.create(w.num_blocks, 2, 128)
    every = torch.arange(w.num_blocks, dtype=torch.int32, device="cuda")
    sel, out = torch.zeros(3, 2, K, dtype=torch.int32, device="cuda"), torch.empty_like(w.q)
    ws, ws2 = pdattn.alloc_workspace(3, 8, 2, 128), pdattn.alloc_select_workspace(3, 2, w.block_table.shape[1])
    pdattn.summarize_pages(w.k_cache, s, every)

    def call():
        pdattn.summarize_append(w.k_cache, s, w.block_table, w.context_lens)
        pdattn.select_pages(w.q, s, w.block_table, w.context_lens, sel, bs, ws2, num_first=1, num_recent=2)
        pdattn.decode_selected(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, sel, w.scale, out, ws)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    w.context_lens.sub_(1)
    w.context_lens_host = w.context_lens_host - 1
    w.q.mul_(-1.5)
    graph.replay()
    table = w.block_table.cpu().numpy()
    want = chosen(w.q.double().cpu().numpy(), s.codes.cpu().numpy(), s.exponents.cpu().numpy(), table, w.context_lens_host, bs, K, 1, 2)
    assert (sel.cpu().numpy() == want).all()
    close(out, *reference(w, want), BF16_WEIGHTS)
    assert pdattn.check(ws) == pdattn.check(ws2) == pdattn.OK


def test_the_bound_holds():
    """The codes enclose every key of the page, so the score bounds its product with the query's codes."""
    NB, d, bs = 40, 64, 16
    k, _ = pool(NB, 1, bs, d, seed=11)
    s = pdattn.PageSummary.create(NB, 1, d)
    pdattn.summarize_pages(k, s, i32(np.arange(NB)))
    # (powers of two by numpy: torch's pow on the GPU gives 0.06249999999999999 for 2.0 ** -4.0)
    w = 2.0 ** s.exponents.double().cpu().numpy()
    lo, hi = (s.codes[:, 0, i].double().cpu().numpy() * w for i in (0, 1))
    x = k[:, 0].double().cpu().numpy()
    assert (lo[:, None] <= x).all() and (x <= hi[:, None]).all()
    # (products of 7 and 8 bits, summed: far below 53 bits; rounding of the sum's last bits is allowed for)
    c = np.random.default_rng(0).integers(-127, 128, d).astype(np.float64)
    bound = np.maximum(c * lo, c * hi).sum(-1)
    assert (bound[:, None] >= (x @ c) * (1 - np.sign(x @ c) * 2.0 ** -40)).all()


def test_wrapper_refuses_what_the_library_cannot_see():
    w = W.make_custom([30, 9], 8, 2, 64, 16, device="cuda:0")
    ws, out, sel = pdattn.alloc_workspace(2, 8, 2, 64), torch.empty_like(w.q), i32(np.zeros((2, 2, 3)))
    args = [w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens]
    s = pdattn.PageSummary.create(w.num_blocks, 2, 64)
    for bad in (sel[:1], sel[:, :1], sel[..., 0], sel.long(), sel.transpose(1, 2)):
        with pytest.raises((ValueError, TypeError)):
            pdattn.decode_selected(*args, bad, w.scale, out, ws)
        with pytest.raises((ValueError, TypeError)):
            pdattn.select_pages(w.q, s, w.block_table, w.context_lens, bad, 16, ws)
    with pytest.raises(pdattn.PdattnError):                               # no recent page
        pdattn.select_pages(w.q, s, w.block_table, w.context_lens, sel, 16, ws, num_recent=0)
    with pytest.raises(ValueError):
        pdattn.summarize_append(w.k_cache[:-1], s, w.block_table, w.context_lens)
    with pytest.raises(ValueError):
        pdattn.summarize_append(w.k_cache, s, w.block_table, w.context_lens, cu_tokens=i32([0, 1, 2]))
    with pytest.raises(ValueError):
        pdattn.summarize_pages(w.k_cache, s, i32([0]), k_scale=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        pdattn.PageSummary(s.codes, s.exponents[:-1])
