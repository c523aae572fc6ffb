"""Prompt attention over the paged cache, with modified scores and masks, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def make(n, L, Hq, Hkv, d, bs, seed=0, nhd=False, sharp=1.0):
    """n[s] new tokens of L[s] per sequence.  Slots past the end and pages that no row references hold NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = np.asarray(n), np.asarray(L)
    N, pages = int(n.sum()), np.maximum(0, -(-L // bs))
    NB, MB = int(pages.sum()) + 2, int(max(1, pages.max())) + 1
    perm = np.random.default_rng(seed).permutation(NB)
    table = np.full((len(n), MB), -7, np.int32)
    shape = (NB, bs, Hkv, d) if nhd else (NB, Hkv, bs, d)
    kc, vc = (torch.randn(*shape, device="cuda", dtype=BF16, generator=g) for _ in range(2))
    if nhd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    used = torch.zeros(NB, bs, dtype=torch.bool, device="cuda")
    at = 0
    for s in range(len(n)):
        table[s, :pages[s]] = perm[at:at + pages[s]]
        at += pages[s]
        for b in range(pages[s]):
            used[table[s, b], :min(bs, L[s] - b * bs)] = True
    for x in (kc, vc):
        x.masked_fill_(~used[:, None, :, None], float("nan"))
    q = (torch.randn(N, Hq, d, device="cuda", generator=g) * sharp).to(BF16)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    return dict(q=q, kc=kc, vc=vc, table=i32(table), lens=i32(L), cu=i32(np.concatenate([[0], np.cumsum(n)])), n=n, L=L, bs=bs,
                tab=table, scale=1.0 / math.sqrt(d))


def reference(c, cap=0.0, slopes=None, window=0, begin=None, prefix=None, bad=()):
    """(output, sum of weight times |v|) in 64 bits; bad: pages whose tokens are left out."""
    N, Hq, d = c["q"].shape
    Hkv, bs = c["kc"].shape[1], c["bs"]
    G = Hq // Hkv
    out, size = np.zeros((N, Hq, d)), np.zeros((N, Hq, d))
    t0 = 0
    for s in range(len(c["n"])):
        n, L = int(c["n"][s]), int(c["L"][s])
        if n == 0:
            continue
        pg = torch.from_numpy(np.clip(c["tab"][s, :-(-max(L, 1) // bs)], 0, c["kc"].shape[0] - 1)).long().cuda()
        pos = torch.arange(L - n, L, device="cuda")
        t = torch.arange(L, device="cuda")
        lo = torch.zeros_like(pos)
        if window:
            lo = (pos - window + 1).clamp(min=0)
        if begin is not None:
            lo = torch.maximum(lo, torch.from_numpy(np.asarray(begin[t0:t0 + n])).long().cuda())
        hi = pos + 1
        if prefix is not None:
            hi = hi.clamp(min=int(prefix[s]))
        hi = torch.where(pos < 0, 0, hi.clamp(max=L))
        seen = (t >= lo[:, None]) & (t < hi[:, None])
        if len(bad):
            here = torch.from_numpy(np.isin(c["tab"][s, t.cpu().numpy() // bs], bad)).cuda()
            seen &= ~here
        for h in range(Hkv):
            k = c["kc"][pg, h].reshape(-1, d)[:L].double()
            v = c["vc"][pg, h].reshape(-1, d)[:L].double()
            x = torch.einsum("ngd,td->gnt", c["q"][t0:t0 + n, h * G:(h + 1) * G].double(), k) * c["scale"]
            if cap:
                x = cap * torch.tanh(x / cap)
            if slopes is not None:
                x = x - slopes[h * G:(h + 1) * G].double().view(-1, 1, 1) * (pos[:, None] - t).abs()
            x = torch.where(seen, x, -math.inf)
            p = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
            v0 = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)
            o = torch.einsum("gnt,td->ngd", p, v0)
            for mark in (math.inf, -math.inf, math.nan):      # what a row sees of non-finite elements decides its output
                m = (v.isnan() if mark != mark else v == mark).double()
                if m.any():
                    hit = torch.einsum("nt,td->nd", seen.double(), m) > 0
                    o = o + torch.where(hit, mark, 0.0)[:, None]
            out[t0:t0 + n, h * G:(h + 1) * G] = o.cpu().numpy()
            size[t0:t0 + n, h * G:(h + 1) * G] = torch.einsum("gnt,td->ngd", p, v0.abs()).cpu().numpy()
        t0 += n
    return out, size


def close(got, want, size):
    # The weights are rounded to bf16 (2^-8 of each at most): 2^-8 of sum p |v|.  The result once more: 2^-8 of it.  Scores and
    # sums in fp32 with exponentials good to 2^-22: below 2^-12 of sum p |v| for scores up to a few hundred.
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    f = np.isfinite(want)
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    err, tol = abs(got[f] - want[f]), 2.0 ** -8 * abs(want[f]) + (2.0 ** -8 + 2.0 ** -12) * size[f] + 1e-30
    assert (err <= tol).all(), (err / tol).max()


def run(c, ws=None, q=None, out=None, **score):
    N, Hq, d = c["q"].shape
    ws = ws if ws is not None else pdattn.alloc_prefill_workspace(len(c["n"]), N, Hq, c["kc"].shape[1], d, c["bs"])
    out = out if out is not None else torch.full_like(c["q"], 7.0)
    pdattn.prefill(c["q"] if q is None else q, c["kc"], c["vc"], c["table"], c["lens"], c["cu"], c["scale"], out, ws,
                   score=pdattn.Score(**score) if score else None)
    assert pdattn.check(ws) == pdattn.OK
    return out


def begins(c, size):
    return np.concatenate([np.arange(L - n, L) // size * size for n, L in zip(c["n"], c["L"])]).astype(np.int32)


@pytest.mark.parametrize("Hq,Hkv,d,bs", [(28, 4, 128, 16), (4, 1, 64, 16), (8, 8, 128, 64), (16, 1, 128, 32), (6, 2, 64, 64),
                                       (5, 1, 128, 16), (13, 1, 64, 32), (9, 1, 128, 64)])
def test_plain_causal(Hq, Hkv, d, bs):
    c = make([1, 0, 37, 300, 5, 130, 0, 64], [1, 40, 37, 300, 700, 131, 0, 1000], Hq, Hkv, d, bs, seed=Hq)
    close(run(c), *reference(c))


@pytest.mark.parametrize("n,L", [([1], [1]), ([1], [129]), ([128], [128]), ([129], [257]), ([2000], [2000]), ([1] * 200, list(range(1, 201))),
                                 ([700, 3], [5000, 20000])])
def test_lengths(n, L):
    c = make(n, L, 14, 2, 128, 16, seed=len(n))
    close(run(c), *reference(c))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias", [(0, True), (30.0, False), (5.0, True)])
@pytest.mark.parametrize("mask", ["causal", "window", "documents", "prefix", "all"])
def test_scores_and_masks(d, cap, bias, mask):
    c = make([200, 1, 33, 400, 90], [200, 77, 400, 900, 300], 6, 2, d, 32, seed=d, sharp=3.0)
    score, ref = {}, {}
    if cap:
        score["logit_cap"] = ref["cap"] = cap
    if bias:
        score["bias_slopes"] = ref["slopes"] = torch.tensor([0.5, 0.2, 0.01, 0.0, -0.001, 1.0], device="cuda")
    if mask in ("window", "all"):
        score["window"] = ref["window"] = 100
    if mask in ("documents", "all"):
        ref["begin"] = begins(c, 90)
        score["key_begin"] = torch.from_numpy(ref["begin"]).cuda()
    if mask in ("prefix", "all"):
        ref["prefix"] = np.array([150, 1000, 0, 450, 300], np.int32)
        score["prefix_lens"] = torch.from_numpy(ref["prefix"]).cuda()
    close(run(c, **score), *reference(c, **ref))


def test_rows_that_see_nothing_and_unordered_documents():
    """First keys drawn at random: many rows see nothing, others a single key; the tiles of a pair need not touch."""
    c = make([150, 260, 40], [150, 500, 2000], 4, 2, 128, 16)
    r = np.random.default_rng(5)
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(c["n"], c["L"])])
    begin = (pos - r.integers(-40, 1500, len(pos)) * (r.random(len(pos)) < 0.8)).astype(np.int32)
    begin[:128] = 5000                                       # a whole tile without keys
    out = run(c, key_begin=torch.from_numpy(begin).cuda())
    want, size = reference(c, begin=begin)
    close(out, want, size)
    assert not out[:128].any()


def test_fewer_keys_than_tokens_and_padding():
    """A sequence with more new tokens than its context: those before position 0 get zeros; rows behind the last sequence
    stay as they are."""
    c = make([10, 200, 3], [4, 150, 3], 8, 2, 64, 16)
    q = torch.cat([c["q"], torch.full((300, 8, 64), float("nan"), device="cuda", dtype=BF16)])
    out = run(c, q=q, out=torch.full_like(q, 7.0))
    close(out[:213], *reference(c))
    assert not out[:6].any() and not out[10:60].any()
    assert bool((out[213:] == 7).all())


def test_negative_and_zero_scale():
    c = make([100, 9], [100, 300], 4, 1, 128, 16)
    for scale in (-0.1, 0.0):
        c["scale"] = scale
        close(run(c), *reference(c))
        close(run(c, logit_cap=2.0), *reference(c, cap=2.0))


def test_values_that_are_not_finite():
    """Infinities and NaN in V reach exactly the rows that see them; in K and in masked places they reach nobody else."""
    c = make([300, 260], [300, 700], 4, 2, 128, 16)
    v, tab = c["vc"], c["tab"]
    for s, t, h, j, x in ((0, 137, 0, 5, math.inf), (0, 200, 1, 100, math.nan), (1, 650, 0, 64, -math.inf), (1, 650, 0, 3, math.inf),
                          (1, 690, 0, 3, -math.inf), (1, 10, 1, 127, math.nan)):
        v[tab[s, t // 16], h, t % 16, j] = x
    close(run(c), *reference(c))
    begin = begins(c, 140)
    close(run(c, key_begin=torch.from_numpy(begin).cuda()), *reference(c, begin=begin))
    # masked keys may be anything
    c["kc"][tab[1, 0:20]] = math.nan
    c["kc"][tab[1, 20:25]] = math.inf
    c["vc"][tab[1, 0:25]] = math.nan
    begin = np.concatenate([np.zeros(300), np.full(260, 400)]).astype(np.int32)
    out = run(c, key_begin=torch.from_numpy(begin).cuda())
    close(out, *reference(c, begin=begin))


def test_a_key_of_nan_reaches_only_those_who_see_it():
    c = make([200], [200], 4, 2, 64, 16)
    want, size = reference(c)
    c["kc"][c["tab"][0, 150 // 16], 0, 150 % 16] = math.nan
    out = run(c)
    close(out[:150], want[:150], size[:150])
    close(out[:, 2:], want[:, 2:], size[:, 2:])
    assert bool(out[150:, :2].isnan().all())


def test_bad_pages_are_left_out_and_reported():
    c = make([100, 64, 30], [300, 64, 90], 4, 2, 128, 16)
    NB = c["kc"].shape[0]
    c["tab"][0, 3], c["tab"][0, 18], c["tab"][1, 2] = NB, -1, NB + 5
    c["table"] = torch.from_numpy(c["tab"]).cuda()
    ws = pdattn.alloc_prefill_workspace(3, 194, 4, 2, 128)
    out = torch.empty_like(c["q"])
    args = (c["q"], c["kc"], c["vc"], c["table"], c["lens"], c["cu"], c["scale"], out, ws)
    pdattn.prefill(*args)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX and pdattn.check(ws) == pdattn.OK
    close(out, *reference(c, bad=(NB, -1, NB + 5)))
    # a context longer than its table row: the tokens past the row are left out, nothing past the row is read
    short = c["table"][:, :10].contiguous()
    c["tab"] = np.concatenate([c["tab"][:, :10], np.full((3, 12), -1, np.int32)], 1)
    pdattn.prefill(c["q"], c["kc"], c["vc"], short, c["lens"], c["cu"], c["scale"], out, ws)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX
    close(out, *reference(c, bad=(NB, -1, NB + 5)))


def test_token_major_pages_and_shared_pages():
    c = make([120, 120], [120, 120], 8, 4, 128, 32, nhd=True)
    close(run(c), *reference(c))
    c = make([50, 50], [300, 300], 8, 4, 128, 16)
    c["tab"][1, :10] = c["tab"][0, :10]
    c["table"] = torch.from_numpy(c["tab"]).cuda()
    close(run(c), *reference(c))


def test_same_bits_every_time_and_under_renumbered_pages():
    c = make([700, 5, 260], [700, 900, 1500], 14, 2, 128, 16)
    score = dict(logit_cap=30.0, bias_slopes=torch.linspace(0, 0.5, 14, device="cuda"))
    a = run(c, **score)
    for _ in range(3):
        assert torch.equal(run(c, **score), a)
    perm = torch.randperm(c["kc"].shape[0], device="cuda")
    c["kc"], c["vc"] = c["kc"][perm].contiguous(), c["vc"][perm].contiguous()
    back = torch.argsort(perm).int()
    c["table"] = torch.where(c["table"] >= 0, back[c["table"].clamp(min=0).long()], c["table"])
    assert torch.equal(run(c, **score), a)


def test_agrees_with_the_decode_step():
    """One new token per sequence is the decode step; several are pdattn_decode_multi's."""
    c = make([1] * 20, np.arange(1, 21) * 37, 8, 2, 128, 16)
    out, other = run(c), torch.empty_like(c["q"])
    ws = pdattn.alloc_workspace(20, 8, 2, 128)
    pdattn.decode_ex(c["q"], c["kc"], c["vc"], c["table"], c["lens"], c["scale"], other, ws)
    want, size = reference(c)
    close(out, want, size)
    assert (abs(out.double() - other.double()).cpu().numpy() <= 2.0 ** -7 * abs(want) + 2.0 ** -7 * size).all()


def test_largest_pool_offsets():
    """Pages past 2^32 elements of a pool."""
    NB, Hkv, bs, d = 300000, 2, 64, 128                     # 4.9e9 elements a cache
    kc, vc = (torch.zeros(NB, Hkv, bs, d, device="cuda", dtype=BF16) for _ in range(2))
    pages = [NB - 1, 3, NB - 2]
    for p in pages:
        kc[p].normal_()
        vc[p].normal_()
    q = torch.randn(70, 4, d, device="cuda").to(BF16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = dict(q=q, kc=kc, vc=vc, table=i32([pages]), lens=i32([190]), cu=i32([0, 70]), n=np.array([70]), L=np.array([190]), bs=bs,
             tab=np.array([pages]), scale=0.1)
    vc[NB - 1, 0, 5, 7] = math.inf
    close(run(c), *reference(c))


def test_captured_replayed_and_on_another_stream():
    c = make([40, 100], [200, 100], 4, 2, 128, 16)
    ws = pdattn.alloc_prefill_workspace(2, 140, 4, 2, 128)
    out = run(c, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pdattn.prefill(c["q"], c["kc"], c["vc"], c["table"], c["lens"], c["cu"], c["scale"], out, ws)
        pdattn.prefill(c["q"], c["kc"], c["vc"], c["table"], c["lens"], c["cu"], c["scale"], out, ws)
    c["cu"][1] = 30                                          # the replayed call goes by the tokens of its time
    c["n"] = np.array([30, 110])
    c["lens"][1] = 110
    c["L"] = np.array([200, 110])
    c["vc"].nan_to_num_(0.0)
    c["kc"].nan_to_num_(0.0)
    graph.replay()
    close(out, *reference(c))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = torch.empty_like(out)
    pdattn.prefill(c["q"], c["kc"], c["vc"], c["table"], c["lens"], c["cu"], c["scale"], other, ws, stream=side)
    side.synchronize()
    assert torch.equal(other, out)


def test_wrapper_refuses_what_the_library_cannot_see():
    c = make([4], [20], 4, 2, 64, 16)
    ws = pdattn.alloc_prefill_workspace(1, 4, 4, 2, 64)
    good = dict(q=c["q"], k_cache=c["kc"], v_cache=c["vc"], block_table=c["table"], context_lens=c["lens"], cu_tokens=c["cu"], scale=1.0,
                out=torch.empty_like(c["q"]), workspace=ws)
    for name, bad in [("q", c["q"].half()), ("cu_tokens", c["cu"].long()), ("k_cache", c["kc"].float())]:
        with pytest.raises(TypeError):
            pdattn.prefill(**dict(good, **{name: bad}))
    for name, bad in [("out", good["out"][:2]), ("cu_tokens", c["cu"][:1]), ("v_cache", c["vc"][:, :1]), ("block_table", c["table"].expand(2, -1)),
                      ("q", c["q"].transpose(0, 1))]:
        with pytest.raises(ValueError):
            pdattn.prefill(**dict(good, **{name: bad}))
    with pytest.raises(ValueError):
        pdattn.prefill(**good, score=pdattn.Score(bias_slopes=torch.zeros(3, device="cuda")))
    with pytest.raises(ValueError):
        pdattn.prefill(**good, score=pdattn.Score(key_begin=torch.zeros(5, dtype=torch.int32, device="cuda")))
    with pytest.raises(pdattn.PdattnError):
        pdattn.prefill(**good, score=pdattn.Score(logit_cap=-1.0))


@pytest.mark.parametrize("n,L,Hq,Hkv,d", [([1], [20000], 4, 1, 128), ([40], [30000], 28, 4, 128), ([5, 0, 17], [9000, 77, 600], 8, 2, 64),
                                         ([100, 3], [100, 15000], 16, 1, 128), ([300], [4000], 2, 2, 64)])
@pytest.mark.parametrize("what", ["causal", "window", "documents", "capped"])
def test_few_tokens_over_long_contexts(n, L, Hq, Hkv, d, what):
    """Cut along the keys: parts of very different worth, some without a visible key."""
    c = make(n, L, Hq, Hkv, d, 16, seed=Hq + d, sharp=2.0)
    score, ref = {}, {}
    if what == "window":
        score["window"] = ref["window"] = 3000
    if what == "documents":
        r = np.random.default_rng(1)
        pos = np.concatenate([np.arange(b - a, b) for a, b in zip(n, L)])
        ref["begin"] = np.maximum(0, pos - r.integers(0, 12000, len(pos))).astype(np.int32)
        ref["begin"][-1] = 30000                             # the last token sees nothing
        score["key_begin"] = torch.from_numpy(ref["begin"]).cuda()
    if what == "capped":
        score["logit_cap"] = ref["cap"] = 8.0
        score["bias_slopes"] = ref["slopes"] = torch.full((Hq,), 0.001, device="cuda")
    want, size = reference(c, **ref)
    out = run(c, **score)
    close(out, want, size)
    assert torch.equal(run(c, **score), out)
    # without room for the parts' results the items stay whole
    small = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    close(run(c, ws=small, **score), want, size)
    some = torch.zeros(8448 + 1024 + 10 * 2 * (d + 2) * 512 + 77, dtype=torch.uint8, device="cuda")
    close(run(c, ws=some, **score), want, size)


def test_cut_items_with_values_that_are_not_finite():
    c = make([20], [12000], 4, 1, 128, 16)
    v, tab = c["vc"], c["tab"]
    for t, j, x in ((50, 3, math.inf), (6000, 3, -math.inf), (7000, 9, math.inf), (11990, 77, math.nan), (11999, 100, -math.inf)):
        v[tab[0, t // 16], 0, t % 16, j] = x
    close(run(c), *reference(c))
    begin = np.linspace(0, 11000, 20).astype(np.int32)
    close(run(c, key_begin=torch.from_numpy(begin).cuda()), *reference(c, begin=begin))


@pytest.mark.parametrize("cap", [1e-6, 0.5, 300.0, 1e4, 1e6])
def test_caps_far_from_the_scores(cap):
    """A cap far above the scores leaves them as they are to fp32 (tanh good to 2^-18 of small values: 2^-14 for scores
    up to 16), one far below makes them all alike."""
    c = make([90, 3], [200, 900], 4, 2, 128, 16, sharp=2.0)
    close(run(c, logit_cap=cap), *reference(c, cap=cap))


def test_lengths_that_no_table_row_can_hold():
    """The largest length there is: the work is bounded by the row, whose tokens all count."""
    c = make([40, 5], [128, 160], 4, 2, 128, 16)
    c["tab"] = c["tab"][:, :8].copy()
    want, size = reference(dict(c, n=np.array([40, 5]), L=np.array([128, 128])), prefix=[128, 128])
    lens = torch.tensor([2 ** 31 - 1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ws = pdattn.alloc_prefill_workspace(2, 45, 4, 2, 128)
    out = torch.empty_like(c["q"])
    pdattn.prefill(c["q"], c["kc"], c["vc"], c["table"][:, :8].contiguous(), lens, c["cu"], c["scale"], out, ws)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX
    close(out, want, size)


def test_cut_items_start_from_any_workspace_contents_and_keep_a_key_of_nan_to_those_who_see_it():
    c = make([30], [9000], 4, 2, 128, 16)
    ws = pdattn.alloc_prefill_workspace(1, 30, 4, 2, 128)
    ws[8448:] = 255                                          # NaN in every part's result
    begin = np.linspace(0, 8990, 30).astype(np.int32)
    dev = torch.from_numpy(begin).cuda()
    want, size = reference(c, begin=begin)
    close(run(c, ws=ws, key_begin=dev), want, size)
    c["kc"][c["tab"][0, 4000 // 16], 0, 4000 % 16] = math.nan
    out = run(c, ws=ws, key_begin=dev)
    sees = begin <= 4000
    close(out[~torch.from_numpy(sees).cuda()], want[~sees], size[~sees])
    close(out[:, 2:], want[:, 2:], size[:, 2:])
    assert bool(out[torch.from_numpy(sees).cuda(), :2].isnan().all())


def test_cut_calls_captured_and_replayed_on_one_workspace():
    """Two graphs that share a workspace, replayed in turn, and a call with other tokens between them."""
    c, e = make([12], [7000], 4, 1, 128, 16), make([50, 2], [900, 5000], 4, 1, 128, 16)
    ws = max((pdattn.alloc_prefill_workspace(len(x["n"]), int(x["n"].sum()), 4, 1, 128) for x in (c, e)), key=len)
    outs, graphs = [run(c, ws=ws), run(e, ws=ws)], []
    keep = [o.clone() for o in outs]
    for x, o in zip((c, e), outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pdattn.prefill(x["q"], x["kc"], x["vc"], x["table"], x["lens"], x["cu"], x["scale"], o, ws)
        graphs.append(graph)
    for _ in range(3):
        for o in outs:
            o.fill_(7.0)
        graphs[1].replay()
        graphs[0].replay()
        assert torch.equal(outs[0], keep[0]) and torch.equal(outs[1], keep[1])
        assert torch.equal(run(e, ws=ws), keep[1])


def test_items_of_very_different_length():
    """One long sequence among many of a token or none: what a CTA draws next is settled while others still work."""
    n = [1] * 150 + [0] * 40 + [700] + [2] * 90 + [0] * 30
    L = [1 + i % 300 for i in range(150)] + [0] * 40 + [20000] + [2 + 40 * i for i in range(90)] + [5] * 30
    c = make(n, L, 14, 2, 128, 16, seed=4)
    close(run(c), *reference(c))
    begin = begins(c, 128)
    close(run(c, key_begin=torch.from_numpy(begin).cuda()), *reference(c, begin=begin))


@pytest.mark.parametrize("n,L", [([8] * 16, [4000 - 200 * i for i in range(16)]), ([700], [3000]), ([30, 0, 1] * 6, [900, 50, 7000] * 6)])
def test_items_that_need_part_of_a_second_round(n, L):
    """Between half and two thirds as many items as CTAs: three parts each, short ones fewer."""
    c = make(n, L, 28, 4, 128, 16, seed=len(n))
    slopes = torch.linspace(0, 0.1, 28, device="cuda")
    out = run(c, bias_slopes=slopes, window=2500)
    close(out, *reference(c, slopes=slopes, window=2500))
    assert torch.equal(run(c, bias_slopes=slopes, window=2500), out)
    small = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    close(run(c, ws=small), *reference(c))


def capped_neighbours(G, cap):
    """Two sequences whose rows share tiles with what nobody may notice: unused slots, a neighbour's queries, padding rows."""
    c = make([9, 40], [150, 300], 2 * G, 2, 128, 16, seed=G, sharp=2.0)
    for x in (c["kc"], c["vc"]):
        x.nan_to_num_(0.0)                               # unused slots: 0 in place of NaN
    return c, dict(logit_cap=cap)


@pytest.mark.parametrize("G", [2, 7])
@pytest.mark.parametrize("cap", [50.0, 1e4, 1e5, 1e6])
@pytest.mark.parametrize("junk", [1e30, math.inf])
def test_capped_scores_do_not_depend_on_what_the_row_does_not_see(G, cap, junk):
    """The same bits whatever lies in unused slots, behind key_begin, in the next sequence's queries, or was left in shared
    memory by an earlier kernel."""
    c, score = capped_neighbours(G, cap)
    begin = np.zeros(49, np.int32)
    begin[:9] = 70
    dev = torch.from_numpy(begin).cuda()
    plain = run(c, key_begin=dev, **score)
    want, size = reference(c, cap=cap, begin=begin)
    close(plain, want, size)
    bs, tab = c["bs"], c["tab"]
    for s, L in ((0, 150), (1, 300)):                    # past the end of each context
        c["kc"][tab[s, (L - 1) // bs], :, L % bs:] = junk
        c["vc"][tab[s, (L - 1) // bs], :, L % bs:] = junk
    c["kc"][tab[0, :4]] = junk                           # keys 0 .. 63: before the first sequence's first key
    c["q"][9:] *= 1e4
    run(make([300], [300], 2 * G, 2, 128, 16, sharp=1e5), logit_cap=1.0)       # large queries in every tile of shared memory
    out = run(c, key_begin=dev, **score)
    assert torch.equal(out[:9], plain[:9])
    close(out[:9], want[:9], size[:9])


@pytest.mark.parametrize("cap", [1e4, 1e5, 1e6])
def test_large_and_small_capped_scores_in_one_tile(cap):
    """A row's small scores keep their precision beside another row's scores past the cap."""
    c = make([64], [300], 4, 2, 128, 16, sharp=2.0)
    c["q"][::5] *= 2e6                                   # every fifth token: scores far past the cap
    want, size = reference(c, cap=cap)
    small = np.arange(64) % 5 != 0
    close(run(c, logit_cap=cap)[torch.from_numpy(small).cuda()], want[small], size[small])


@pytest.mark.parametrize("cap", [1e4, 3e4, 1e5, 1e6])
@pytest.mark.parametrize("X", [8192.0, -8192.0])
def test_large_caps_keep_large_scores(cap, X):
    """Two keys whose logits agree: a score of X whose bias takes the capped score away, and a score of 0.  With v = 1 and -1 the
    output is tanh of half the logits' error.  Roundings of the first logit, in units of 2^-24 of it: tanh 8 (2^-21), its argument
    2, cap and product 3, slope 2, their sum 1; 24 are allowed for.  The weights are rounded to bf16: 2^-9 of each at most."""
    d = 128
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, kc, vc = (torch.zeros(s, device="cuda", dtype=BF16) for s in ((1, 2, d), (1, 1, 16, d), (1, 1, 16, d)))
    q[..., 3], kc[0, 0, 0, 3] = X / 64, 64.0
    vc[0, 0, 0], vc[0, 0, 1] = 1.0, -1.0
    c = dict(q=q, kc=kc, vc=vc, table=i32([[0]]), lens=i32([2]), cu=i32([0, 1]), n=[1], L=[2], bs=16, scale=1.0)
    capped = cap * math.tanh(X / cap)
    out = run(c, logit_cap=cap, bias_slopes=torch.full((2,), capped, device="cuda"))
    assert float(out.float().abs().max()) <= 12 * 2.0 ** -24 * abs(X) + 2.0 ** -8


@pytest.mark.parametrize("d,Hq", [(64, 2), (128, 6)])
def test_second_tiles_that_come_and_go_beside_values_that_are_not_finite(d, Hq):
    """Items of one and of two tiles in turn, many to a CTA, masks and non-finite values in most of their key tiles."""
    r = np.random.default_rng(11)
    S = 420
    n = np.where(np.arange(S) % 3 == 0, r.integers(1, 260, S), r.integers(1, 60, S))
    L = n + r.integers(0, 1400, S)
    c = make(n, L, Hq, 2, d, 16, seed=d)
    for s in range(S):
        for t in r.integers(0, L[s], 3):
            c["vc"][c["tab"][s, t // 16], int(r.integers(0, 2)), t % 16, int(r.integers(0, d))] = float(r.choice([math.inf, -math.inf, math.nan]))
    pos = np.concatenate([np.arange(b - a, b) for a, b in zip(n, L)])
    begin = np.maximum(0, pos - r.integers(0, 1200, len(pos))).astype(np.int32)
    want, size = reference(c, begin=begin)
    dev = torch.from_numpy(begin).cuda()
    for _ in range(3):
        close(run(c, key_begin=dev), want, size)


@pytest.mark.parametrize("L,key", [(600, 5), (600, 560), (600, 300), (9000, 40), (9000, 8900)])
def test_a_visible_infinity_of_vanishing_weight_is_never_lost(L, key):
    """A steep bias: the weight of a far key is 0 in 32 bits.  Whatever tile it lies in, what sees it is not finite and nothing else
    is touched."""
    n = 90
    c = make([n], [L], 4, 2, 128, 16)
    c["vc"][c["tab"][0, key // 16], 0, key % 16, 9] = math.inf
    slopes = torch.full((4,), 3.0, device="cuda")
    out = run(c, bias_slopes=slopes)
    c["vc"][c["tab"][0, key // 16], 0, key % 16, 9] = 0.0
    want, size = reference(c, slopes=slopes)
    sees = torch.arange(L - n, L) >= key
    hit = torch.zeros(out.shape, dtype=torch.bool)
    hit[sees, :2, 9] = True
    assert not out.cpu()[hit].isfinite().any()
    o = out.clone()
    o[hit.cuda()] = 0.0
    want[hit.numpy()] = 0.0
    close(o, want, size)
