"""Speculative and sparse decoding over the paged cache, as cases that can be timed: attention for a tree of drafted
tokens, taking the accepted path over, page summaries, the choice of pages by them, and attention over chosen pages.

`run` computes them in plain torch operations, or with `own` set through paper_2607_09207_b200.pdattn."""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------
def _case(op, **kw):
    c = dict(op=op, Hq=28, Hkv=4, d=128, bs=16, fp8=False, shape=1, S=4, n_lo=1, n_hi=1, h_lo=0, h_hi=100)
    if op in ("select", "selected"):
        c.update(K=64, first=1, recent=2)
    c.update(kw)
    return c


def listed():
    return [
        # a handful of short sequences with a few drafted tokens each
        _case("tree", name="tree tiny", n_hi=7, h_hi=255, Hq=4, Hkv=1, d=64),
        # the 7B-shaped rollout batch verifying a small tree per sequence
        _case("tree", name="tree 256x8", S=256, n_lo=5, n_hi=8, h_lo=512, h_hi=4600),
        # a late rollout: few long sequences are left, each with a large tree
        _case("tree", name="tree 8x64 long", S=8, n_lo=57, n_hi=64, h_lo=8000, h_hi=32000, Hq=64, Hkv=8, bs=64),
        # long contexts over an fp8 cache, sixteen tokens each
        _case("tree", name="tree fp8 32x16", S=32, n_lo=9, n_hi=16, h_lo=1000, h_hi=32767, Hq=64, Hkv=8, bs=32, fp8=True),
        # the accepted paths of the 7B-shaped batch taken over, rejected pages given back
        _case("accept", name="accept 256x8", S=256, n_lo=5, n_hi=8, h_lo=512, h_hi=1800),
        # large trees over an fp8 cache
        _case("accept", name="accept fp8 48x64", S=48, n_lo=33, n_hi=64, h_lo=100, h_hi=3000, Hq=64, Hkv=8, bs=32, fp8=True),
        # prompts that have just been appended: all their whole pages summarised
        _case("summarize", name="summarize prompts", S=12, n_lo=700, n_hi=2100, h_hi=0, Hq=40, Hkv=8),
        # one decode step: one sequence in sixteen fills a page
        _case("summarize", name="summarize decode 256x1", S=256, h_lo=512, h_hi=2000),
        # long contexts: 128 pages of up to 2048 chosen for each KV head
        _case("select", name="select 48 long", S=48, h_lo=1000, h_hi=32767, Hq=64, Hkv=8, K=128, first=1, recent=4),
        # a small batch
        _case("select", name="select 6 small", S=6, h_lo=100, h_hi=4000, K=32),
        # the attention that follows: 2048 of up to 32,768 tokens
        _case("selected", name="selected 48 long", S=48, h_lo=1000, h_hi=32767, Hq=64, Hkv=8, K=128, first=1, recent=4),
        # the 7B-shaped batch over an fp8 cache with pages of 32
        _case("selected", name="selected fp8 256", S=256, h_lo=512, h_hi=8703, bs=32, K=32, fp8=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "accept", "summarize", "select", "select", "selected", "selected"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16])
    d = rng.choice([64, 128, 128])
    kw = dict(Hkv=Hkv, Hq=Hkv * G, d=d, bs=rng.choice([16, 32, 64]), shape=rng.randrange(1 << 20), fp8=rng.random() < 0.4)
    if op == "tree":
        n, h = _log(rng, 1, 64), _log(rng, 1, 20000)
        S = max(1, min(_log(rng, 1, 300), int(1.2e6 / (h * Hkv * max(1.0, n * G / 128)))))
        kw.update(S=S, n_lo=max(1, n // 3), n_hi=n, h_lo=h // 6, h_hi=h)
    elif op == "accept":
        kw.update(S=_log(rng, 1, 256), n_lo=1, n_hi=_log(rng, 1, 64), h_lo=0, h_hi=_log(rng, 1, 2000))
    elif op == "summarize":
        if rng.random() < 0.3:          # single tokens, few of which fill a page
            kw.update(S=rng.randrange(150, 300), bs=16, h_hi=_log(rng, 100, 2000))
        else:
            S = _log(rng, 1, 150)
            n = _log(rng, 2 * kw["bs"], 20000 // S)
            kw.update(S=S, n_lo=n // 2, n_hi=n, h_lo=0, h_hi=_log(rng, 1, 2000))
    else:
        h = _log(rng, 16 * kw["bs"], 30000)
        S = max(1, min(_log(rng, 1, 400), int(6e6 / (h * Hkv))))
        K = _log(rng, 3, max(4, h // (4 * kw["bs"])))
        kw.update(S=S, h_lo=h // 2, h_hi=h, K=K, first=rng.choice([0, 1, min(4, K - 2)]), recent=rng.choice([1, 2]))
        if op == "selected":
            kw["h_lo"] = h // 6
            kw.update(S=max(1, min(S, int(1.5e6 / (min(h, K * kw["bs"]) * Hkv)))))
    return _case(op, **kw)


def _shape(c):
    """New tokens and context lengths (new tokens included) of the case's sequences (the case alone decides them)."""
    r = np.random.default_rng(c["shape"])
    n = r.integers(c["n_lo"], c["n_hi"] + 1, c["S"])
    return n.astype(np.int64), (r.integers(min(c["h_lo"], c["h_hi"]), c["h_hi"] + 1, c["S"]) + n).astype(np.int64)


def _width(n):
    """Tokens of a level of a drafted tree of n tokens: about as many levels as a level has tokens."""
    return int(math.ceil(math.sqrt(n)))


def work(c):
    n, L = _shape(c)
    N, eb, G = int(n.sum()), 1 if c["fp8"] else 2, c["Hq"] // c["Hkv"]
    row = c["Hkv"] * c["d"] * eb                      # a token's K, or V
    pages = -(-L // c["bs"])
    if c["op"] == "tree":
        return {"bytes": int(L.sum()) * 2 * row + N * c["Hq"] * c["d"] * 4 + 8 * N, "flops": 4 * c["d"] * c["Hq"] * int((n * L).sum())}
    if c["op"] == "accept":
        path = sum(-(-int(x) // _width(x)) for x in n) / 2           # half of the longest path on average, written and read
        return {"bytes": int(path * 4 * row) + 8 * int(pages.sum()), "flops": 0}
    if c["op"] == "summarize":
        full = int((L // c["bs"] - (L - n) // c["bs"]).sum())
        return {"bytes": full * (c["bs"] * row + c["Hkv"] * (2 * c["d"] + 1)), "flops": 2 * full * c["bs"] * c["Hkv"] * c["d"]}
    seen = np.minimum(pages, c["K"])
    if c["op"] == "select":
        scored = np.where(pages > c["K"], pages - c["first"] - c["recent"], 0)
        scored = int(scored.sum()) * c["Hkv"]
        return {"bytes": scored * (2 * c["d"] + 1) + c["S"] * (c["Hq"] * c["d"] * 2 + c["Hkv"] * c["K"] * 4),
                "flops": scored * 4 * c["d"] * G}
    tokens = int(np.where(pages <= c["K"], L, (seen - 1) * c["bs"] + (L - 1) % c["bs"] + 1).sum())
    return {"bytes": tokens * 2 * row + c["S"] * (c["Hq"] * c["d"] * 4 + c["Hkv"] * c["K"] * 4),
            "flops": 4 * c["d"] * c["Hq"] * tokens}


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _trees(n, seed):
    """Parents of drafted trees in levels (every token of a level continues one of the level before), their masks, and one
    path from a root down for each.  The paths start at token 0 or past their own length."""
    r = np.random.default_rng(seed)
    masks, paths = [], []
    for x in n.tolist():
        w, parent = _width(x), []
        for j in range(x):
            parent.append(-1 if j < w else j // w * w - w + int(r.integers(0, w)))
        m = []
        for j in range(x):
            m.append((m[parent[j]] if parent[j] >= 0 else 0) | 1 << j)
        masks += m
        j, path = int(r.integers(0, x)), []
        while j >= 0:
            path.append(j)
            j = parent[j]
        path.reverse()
        if 0 < path[0] < len(path):
            path[0] = 0
        paths.append(path)
    masks = np.array(masks, dtype=np.uint64).view(np.int64)
    depth = max(-(-int(x) // _width(x)) for x in n)
    table = np.full((len(n), depth), -1, np.int32)
    for s, p in enumerate(paths):
        table[s, :len(p)] = p
    return masks, table, np.array([len(p) for p in paths], np.int32)


def _power(a, lo=-40, hi=40):
    """The smallest e in lo .. hi with a <= 127 * 2^e (hi where there is none)."""
    m, k = torch.frexp(a)
    e = k - 7 + (m > 0.9921875).to(k.dtype)
    return torch.where(a == 0, lo, e.clamp(lo, hi))


def _scaled(x, e):
    """x * 2^-e, without a rounding."""
    return x * torch.exp2(-e.float())


def _summary(x):
    """Codes and exponents of pages x [..., slots, d] in 32 bits."""
    lo, hi = x.amin(-2), x.amax(-2)
    fin = torch.isfinite(x).flatten(-2).all(-1)
    lo, hi = (torch.where(fin[..., None], y, 0.0) for y in (lo, hi))
    e = _power(torch.maximum(lo.abs(), hi.abs()).amax(-1))
    codes = torch.stack((torch.floor(_scaled(lo, e[..., None])), torch.ceil(_scaled(hi, e[..., None]))), -2)
    return codes.clamp(-127, 127).to(torch.int8), torch.where(fin, e, 127).to(torch.int8)


def prepare(c, seed):
    from types import SimpleNamespace
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = _shape(c)
    S, Hq, Hkv, d, bs = c["S"], c["Hq"], c["Hkv"], c["d"], c["bs"]
    pages = -(-L // bs)
    total, MB = int(pages.sum()), int(pages.max())
    perm = np.random.default_rng(seed).permutation(total)
    NB = total + 3
    table = np.full((S, MB), -1, np.int32)
    table[np.arange(MB)[None, :] < pages[:, None]] = perm
    st = SimpleNamespace(c=c, scale=1.0 / math.sqrt(d))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", dtype=BF16, generator=g)

    N = int(n.sum())
    st.lens_host, st.n_max, st.N = L.astype(np.int32), int(n.max()), N
    st.cu = _i32(np.concatenate([[0], np.cumsum(n)]))
    if c["op"] != "accept":
        st.table, st.lens = _i32(table), _i32(L)
    if c["op"] == "select":
        # summaries of keys whose channels and pages have means of their own
        st.codes = torch.empty(NB, Hkv, 2, d, dtype=torch.int8, device="cuda")
        st.exps = torch.empty(NB, Hkv, dtype=torch.int8, device="cuda")
        mean = 2 * torch.randn(Hkv, 1, d, device="cuda", generator=g)
        for a in range(0, NB, 4096):
            b = min(NB, a + 4096)
            k = mean + torch.randn(b - a, Hkv, 1, d, device="cuda", generator=g) + normal(b - a, Hkv, bs, d)
            st.codes[a:b], st.exps[a:b] = _summary(k.to(BF16).float())
        st.q = normal(S, Hq, d)
        st.selected = torch.empty(S, Hkv, c["K"], dtype=torch.int32, device="cuda")
        st.ws = torch.zeros(16384 + 8 * S * Hkv * (MB + 64), dtype=torch.uint8, device="cuda")
        return st
    st.k_cache, st.v_cache = normal(NB, Hkv, bs, d), normal(NB, Hkv, bs, d)
    if c["fp8"]:
        st.k_scale = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
        st.v_scale = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
        st.k_cache = (st.k_cache.float() / st.k_scale.view(1, -1, 1, 1)).to(F8).view(torch.uint8)
        st.v_cache = (st.v_cache.float() / st.v_scale.view(1, -1, 1, 1)).to(F8).view(torch.uint8)
        st.v_cache = st.v_cache.transpose(2, 3).contiguous()
    if c["op"] == "summarize":
        st.codes = torch.zeros(NB, Hkv, 2, d, dtype=torch.int8, device="cuda")
        st.exps = torch.zeros(NB, Hkv, dtype=torch.int8, device="cuda")
        st.one = bool((n == 1).all())
        return st
    if c["op"] == "tree":
        st.q = normal(N, Hq, d)
        st.out = torch.zeros_like(st.q)
        masks, _, _ = _trees(n, seed)
        st.mask = torch.from_numpy(masks).cuda()
        st.ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        return st
    if c["op"] == "accept":
        _, path, count = _trees(n, seed)
        st.path, st.count = _i32(path), _i32(count)
        st.new_lens = _i32(L - n + count)
        # the bookkeeping of the pool in one buffer, so that a pass can start from the same books with one copy
        ref = np.zeros(NB, np.int32)
        ref[perm] = 1
        unused = np.flatnonzero(ref == 0)[::-1]
        free = np.full(NB, -1, np.int32)
        free[:len(unused)] = unused
        st.books0 = _i32(np.concatenate([table.reshape(-1), L, ref, free, [len(unused)]]))
        st.books = st.books0.clone()
        parts = torch.split(st.books, [S * MB, S, NB, NB, 1])
        st.table, st.lens, st.ref, st.free, st.free_count = parts[0].view(S, MB), *parts[1:]
        st.books_ws = torch.zeros(16 * NB + 32768, dtype=torch.uint8, device="cuda")
        return st
    st.q = normal(S, Hq, d)
    st.out = torch.zeros_like(st.q)
    # the first and the latest pages and a random choice of the others, in ascending order
    rank = torch.rand(S, Hkv, MB, device="cuda", generator=g)
    b, np_ = torch.arange(MB, device="cuda"), torch.from_numpy(pages).cuda()[:, None, None]
    rank = torch.where((b < c["first"]) | (b >= np_ - c["recent"]), 2.0, rank)
    rank = torch.where(b < np_, rank, -1.0)
    k = min(MB, c["K"])
    top = rank.topk(k, -1)
    at = torch.where(top.values >= 0, top.indices, 1 << 30).sort(-1).values
    st.selected = torch.full((S, Hkv, c["K"]), -1, dtype=torch.int32, device="cuda")
    st.selected[..., :k] = torch.where(at < 1 << 30, at, -1).int()
    st.ws = torch.zeros(16 * S + (64 << 20), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------------------------------------------
def _pieces(count, each, limit=1 << 28):
    """Ranges of the sequences whose intermediate values (`each` elements a sequence) stay below the limit."""
    step = max(1, int(limit // max(1, each)))
    return [(a, min(count, a + step)) for a in range(0, count, step)]


def _pages(st, at, heads=None):
    """K and V of the pages `at` ([S, P] for all heads, or [S, Hkv, P] for one head each), in 32 bits: [S, Hkv, P * bs, d]."""
    c = st.c
    f8 = c["fp8"]
    if at.dim() == 2:
        k, v = st.k_cache[at], st.v_cache[at]                          # [S, P, Hkv, ...]
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    else:
        h = torch.arange(c["Hkv"], device="cuda")[None, :, None]
        k, v = st.k_cache[at, h], st.v_cache[at, h]                    # [S, Hkv, P, ...]
    if f8:
        k = k.view(F8).float() * st.k_scale.view(1, -1, 1, 1, 1)
        v = v.view(F8).float().transpose(3, 4) * st.v_scale.view(1, -1, 1, 1, 1)
    shape = (k.shape[0], c["Hkv"], -1, c["d"])
    return k.float().reshape(shape), v.float().reshape(shape)


def _softmax(x):
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == float("-inf"), 0.0, m))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0)


def _plain_tree(st):
    c, n = st.c, st.n_max
    S, Hq, Hkv, d, G = c["S"], c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    cu, lens = st.cu.long(), st.lens.long()
    tok = torch.arange(st.q.shape[0], device="cuda")
    s_of = torch.searchsorted(cu, tok, right=True) - 1
    j_of = tok - cu[s_of]
    q = torch.zeros(S, n, Hq, d, device="cuda")
    q[s_of, j_of] = st.q.float() * st.scale
    mask = torch.zeros(S, n, dtype=torch.int64, device="cuda")
    mask[s_of, j_of] = st.mask
    out = torch.empty_like(q)
    keys = st.table.shape[1] * c["bs"]
    t = torch.arange(keys, device="cuda")
    for a, b in _pieces(S, keys * Hkv * (G * n + 2 * d)):
        k, v = _pages(st, st.table[a:b].clamp(min=0).long())
        x = q[a:b].view(b - a, n, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(b - a, Hkv, G * n, d)
        x = torch.matmul(x, k.transpose(2, 3)).view(b - a, Hkv, G, n, -1)
        i = t - (lens[a:b] - (cu[a + 1:b + 1] - cu[a:b]))[:, None]     # tree index of each key, negative: history
        bit = (mask[a:b, :, None] >> i.clamp(0, 63)[:, None, :]) & 1
        seen = (i < 0)[:, None, :] | ((bit == 1) & (t < lens[a:b, None])[:, None, :])
        p = _softmax(torch.where(seen[:, None, None], x, float("-inf")))
        o = torch.matmul(p.view(b - a, Hkv, G * n, -1), v)
        out[a:b] = o.view(b - a, Hkv, G, n, d).permute(0, 3, 1, 2, 4).reshape(b - a, n, Hq, d)
    return [out[s_of, j_of].to(BF16)]


def _plain_accept(st):
    c, bs = st.c, st.c["bs"]
    n = (st.cu[1:] - st.cu[:-1]).long()
    base = st.lens.long() - n
    i = torch.arange(st.path.shape[1], device="cuda")
    # (a place past the end of its path is moved onto itself: the last accepted token)
    i = torch.minimum(i[None, :], st.count.long()[:, None] - 1)
    src = base[:, None] + st.path.long().gather(1, i)
    dst = base[:, None] + i
    sp, dp = (st.table.gather(1, x // bs).long() for x in (src, dst))
    st.k_cache[dp, :, dst % bs] = st.k_cache[sp, :, src % bs]
    if c["fp8"]:
        st.v_cache[dp, :, :, dst % bs] = st.v_cache[sp, :, :, src % bs]
    else:
        st.v_cache[dp, :, dst % bs] = st.v_cache[sp, :, src % bs]
    # the pages past the new lengths go back
    cols = torch.arange(st.table.shape[1], device="cuda")
    gone = (cols >= (-(-st.new_lens // bs))[:, None]) & (cols < (-(-st.lens // bs))[:, None])
    st.ref.index_add_(0, st.table.clamp(min=0).view(-1).long(), -gone.view(-1).int())
    st.table[:] = torch.where(gone, -1, st.table)
    st.lens[:] = st.new_lens
    # free pages in descending order of their number, -1 behind them
    free = st.ref == 0
    m = free.sum()
    ids = torch.arange(len(free), device="cuda")
    at = torch.where(free, m - torch.cumsum(free, 0), m + torch.cumsum(~free, 0) - 1)
    st.free[at] = torch.where(free, ids, -1).int()
    st.free_count[0] = m
    caches = [x.view(F8) if c["fp8"] else x for x in (st.k_cache, st.v_cache)]
    return [st.books, *caches]


def _plain_summarize(st):
    bs = st.c["bs"]
    n = st.cu[1:] - st.cu[:-1]
    cols = torch.arange(st.table.shape[1], device="cuda")
    filled = (cols >= ((st.lens - n) // bs)[:, None]) & (cols < (st.lens // bs)[:, None])
    page = st.table[filled].long()
    x = st.k_cache[page]
    x = x.view(F8).float() * st.k_scale.view(1, -1, 1, 1) if st.c["fp8"] else x.float()
    st.codes[page], st.exps[page] = _summary(x)
    return [st.codes, st.exps]


def _plain_select(st):
    c = st.c
    S, Hkv, d, K, G = c["S"], c["Hkv"], c["d"], c["K"], c["Hq"] // c["Hkv"]
    q = st.q.float()
    fin = torch.isfinite(q).all(-1)
    q = torch.where(fin[..., None], q, 0.0)
    eq = _power(q.abs().amax(-1))
    q = torch.round(_scaled(q, eq[..., None])).clamp(-127, 127)
    q = torch.cat((q.clamp(max=0), q.clamp(min=0)), -1).view(S, Hkv, G, 2 * d)      # against the minima, the maxima
    MB = st.table.shape[1]
    pages = -(-st.lens.long() // c["bs"])
    b = torch.arange(MB, device="cuda")
    out = torch.full((S, Hkv, K), -1, dtype=torch.int32, device="cuda")
    for lo, hi in _pieces(S, MB * Hkv * (2 * d + G)):
        at = st.table[lo:hi].clamp(min=0).long()
        codes = st.codes[at].float().view(hi - lo, MB, Hkv, 2 * d).permute(0, 2, 3, 1)
        e = st.exps[at].permute(0, 2, 1)[:, :, None, :].long()                      # [S, Hkv, 1, MB]
        x = torch.matmul(q[lo:hi], codes) * torch.exp2((e + eq[lo:hi].view(hi - lo, Hkv, G, 1)).float())
        x = torch.where(fin[lo:hi].view(hi - lo, Hkv, G, 1), x, float("-inf"))
        x = torch.where(e == 127, float("inf"), x).amax(2)
        np_ = pages[lo:hi, None, None]
        kept = (b < c["first"]) | (b >= np_ - c["recent"])
        # three ranks: kept in any case, by score, past the end; equal scores in ascending order of the page
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices
        rank = torch.where(b >= np_, 2, torch.where(kept, 0, 1)).expand(-1, Hkv, -1).gather(2, order)
        order = order.gather(2, torch.sort(rank, dim=-1, stable=True).indices)[..., :K]
        order = torch.where(order < np_, order, MB).sort(-1).values
        out[lo:hi, :, :order.shape[2]] = torch.where(order < MB, order, -1).int()
    return [out]


def _plain_selected(st):
    c = st.c
    S, Hq, Hkv, d, G, bs = c["S"], c["Hq"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"], c["bs"]
    out = torch.empty(S, Hq, d, device="cuda")
    slot = torch.arange(bs, device="cuda")
    for a, b in _pieces(S, c["K"] * bs * Hkv * (G + 2 * d)):
        sel = st.selected[a:b].long()
        at = st.table[a:b, None, :].expand(-1, Hkv, -1).gather(2, sel.clamp(min=0)).long()
        k, v = _pages(st, at)
        x = torch.matmul(st.q[a:b].float().view(b - a, Hkv, G, d) * st.scale, k.transpose(2, 3))
        seen = (sel >= 0)[..., None] & (sel[..., None] * bs + slot < st.lens.long()[a:b, None, None, None])
        p = _softmax(torch.where(seen.flatten(2)[:, :, None], x, float("-inf")))
        out[a:b] = torch.matmul(p, v).view(b - a, Hq, d)
    return [out.to(BF16)]


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def run(st):
    op = st.c["op"]
    if op == "accept":
        st.books.copy_(st.books0)       # every pass starts from the same books
    if own:
        return _own(st)
    return {"tree": _plain_tree, "accept": _plain_accept, "summarize": _plain_summarize, "select": _plain_select,
            "selected": _plain_selected}[op](st)


def _own(st):
    from paper_2607_09207_b200 import pdattn
    c = st.c
    scales = (st.k_scale, st.v_scale) if c["fp8"] and c["op"] != "select" else ()
    if c["op"] == "tree":
        call = pdattn.decode_tree_fp8 if c["fp8"] else pdattn.decode_tree
        call(st.q, st.k_cache, st.v_cache, *scales, st.table, st.lens, st.cu, st.mask, st.scale, st.out, st.ws,
             max_tree_tokens=st.n_max)
        return [st.out]
    if c["op"] == "accept":
        pool = pdattn.PagePool(st.ref, st.free, st.free_count)
        pdattn.tree_accept(st.k_cache, st.v_cache, st.table, st.lens, st.cu, st.path, st.count)
        pdattn.pages_trim(pool, st.table, st.lens, st.new_lens, c["bs"], st.books_ws)
        caches = [x.view(F8) if c["fp8"] else x for x in (st.k_cache, st.v_cache)]
        return [st.books, *caches]
    if c["op"] == "summarize":
        summary = pdattn.PageSummary(st.codes, st.exps)
        pdattn.summarize_append(st.k_cache, summary, st.table, st.lens, cu_tokens=None if st.one else st.cu,
                                num_tokens=st.N, k_scale=st.k_scale if c["fp8"] else None)
        return [st.codes, st.exps]
    if c["op"] == "select":
        pdattn.select_pages(st.q, pdattn.PageSummary(st.codes, st.exps), st.table, st.lens, st.selected, c["bs"], st.ws,
                            num_first=c["first"], num_recent=c["recent"])
        return [st.selected]
    call = pdattn.decode_selected_fp8 if c["fp8"] else pdattn.decode_selected
    call(st.q, st.k_cache, st.v_cache, *scales, st.table, st.lens, st.selected, st.scale, st.out, st.ws,
         context_lens_host=st.lens_host)
    return [st.out]


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(c, seed):
    st = prepare(c, seed)
    n, L = _shape(c)
    table = st.table.cpu().numpy().astype(np.int64)
    cu = np.concatenate([[0], np.cumsum(n)])
    return {"tree": _exact_tree, "accept": _exact_accept, "summarize": _exact_summarize, "select": _exact_select,
            "selected": _exact_selected}[c["op"]](c, st, n, L, table, cu)


def _head(c, st, at, h):
    """K and V of the pages `at` for KV head h, in 64 bits: [tokens, d]."""
    D = torch.float64
    if c["fp8"]:
        return (st.k_cache[at, h].view(F8).to(D).reshape(-1, c["d"]) * st.k_scale[h].to(D),
                st.v_cache[at, h].view(F8).to(D).mT.reshape(-1, c["d"]) * st.v_scale[h].to(D))
    return st.k_cache[at, h].to(D).reshape(-1, c["d"]), st.v_cache[at, h].to(D).reshape(-1, c["d"])


def _exact_tree(c, st, n, L, table, cu):
    G, D = c["Hq"] // c["Hkv"], torch.float64
    out = torch.empty(st.q.shape, dtype=D, device="cuda")
    masks = st.mask.cpu().numpy().view(np.uint64)
    for s in range(c["S"]):
        at = torch.from_numpy(table[s, :-(-int(L[s]) // c["bs"])]).cuda()
        span, h0 = slice(int(cu[s]), int(cu[s + 1])), int(L[s] - n[s])
        hidden = np.zeros((n[s], L[s]), bool)
        hidden[:, h0:] = (masks[span, None] >> np.arange(n[s], dtype=np.uint64)) & np.uint64(1) == 0
        hidden = torch.from_numpy(hidden).cuda()
        for h in range(c["Hkv"]):
            k, v = (x[:int(L[s])] for x in _head(c, st, at, h))
            y = torch.einsum("jgd,td->gjt", st.q[span, h * G:h * G + G].to(D), k) * st.scale
            y.masked_fill_(hidden, -math.inf)
            out[span, h * G:h * G + G] = torch.einsum("gjt,td->jgd", torch.softmax(y, -1), v)
    return [out]


def _exact_accept(c, st, n, L, table, cu):
    bs = c["bs"]
    k, v = ((x.view(F8) if c["fp8"] else x).double() for x in (st.k_cache, st.v_cache))
    if c["fp8"]:
        v = v.mT.contiguous()
    path, count = st.path.cpu().numpy(), st.count.cpu().numpy()
    ref, lens = st.ref.cpu().numpy(), st.lens.cpu().numpy()
    for s in range(c["S"]):
        at = int(L[s] - n[s])
        took = [at + int(x) for x in path[s, :count[s]]]
        place = [at + i for i in range(count[s])]
        a, b, x, y = (torch.tensor(z, device="cuda") for z in ([table[s, t // bs] for t in took], [t % bs for t in took],
                                                              [table[s, t // bs] for t in place], [t % bs for t in place]))
        k[x, :, y], v[x, :, y] = k[a, :, b], v[a, :, b]
        lens[s] = at + count[s]
        for p in range(-(-int(lens[s]) // bs), -(-int(L[s]) // bs)):
            ref[table[s, p]] -= 1
            table[s, p] = -1
    unused = np.flatnonzero(ref == 0)[::-1]
    free = np.full(len(ref), -1, np.int32)
    free[:len(unused)] = unused
    if c["fp8"]:
        v = v.mT.contiguous()
    return [np.concatenate([table.reshape(-1), lens, ref, free, [len(unused)]]).astype(np.int32), k, v]


def _exact_summarize(c, st, n, L, table, cu):
    codes, exps = st.codes.cpu().numpy().copy(), st.exps.cpu().numpy().copy()
    keys = st.k_cache
    scale = st.k_scale.cpu().numpy() if c["fp8"] else np.ones(c["Hkv"], np.float32)
    for s in range(c["S"]):
        at = table[s, int(L[s] - n[s]) // c["bs"]:int(L[s]) // c["bs"]]
        if not len(at):
            continue
        x = keys[torch.from_numpy(at).cuda()]
        x = (x.view(F8) if c["fp8"] else x).float().cpu().numpy() * scale[None, :, None, None]     # (a 32-bit product by definition)
        x = x.astype(np.float64)
        lo, hi = x.min(2), x.max(2)
        top = np.maximum(-lo, hi).max(-1)
        e = np.full(top.shape, -40)
        while (top > 127 * 2.0 ** e)[e < 40].any():
            e = np.where((top > 127 * 2.0 ** e) & (e < 40), e + 1, e)
        w = 2.0 ** e[..., None]
        codes[at, :, 0] = np.clip(np.floor(lo / w), -127, 127)
        codes[at, :, 1] = np.clip(np.ceil(hi / w), -127, 127)
        exps[at] = e
    return [codes, exps]


def _exact_select(c, st, n, L, table, cu):
    G, K = c["Hq"] // c["Hkv"], c["K"]
    q = st.q.double().cpu().numpy()
    codes, exps = st.codes.cpu().numpy(), st.exps.cpu().numpy()
    out = np.full((c["S"], c["Hkv"], K), -1, np.int32)
    for s in range(c["S"]):
        P = -(-int(L[s]) // c["bs"])
        for h in range(c["Hkv"]):
            if P <= K:
                out[s, h, :P] = np.arange(P)
                continue
            at = table[s, :P]
            box = codes[at, h].astype(np.int64)                       # [P, 2, d]
            best = np.full(P, -np.inf)
            for i in range(h * G, h * G + G):
                top, e = np.abs(q[s, i]).max(), -40
                while top > 127 * 2.0 ** e and e < 40:
                    e += 1
                z = np.clip(np.rint(q[s, i] / 2.0 ** e), -127, 127).astype(np.int64)
                dot = np.where(z > 0, box[:, 1], box[:, 0]) @ z
                best = np.maximum(best, dot * 2.0 ** (exps[at, h].astype(np.float64) + e))
            must = list(range(c["first"])) + list(range(P - c["recent"], P))
            rest = [int(b) for b in np.lexsort((np.arange(P), -best)) if b not in must]
            out[s, h] = sorted(must + rest[:K - len(must)])
    return [out]


def _exact_selected(c, st, n, L, table, cu):
    G, D, bs = c["Hq"] // c["Hkv"], torch.float64, c["bs"]
    out = torch.empty(st.q.shape, dtype=D, device="cuda")
    chosen = st.selected.cpu().numpy()
    for s in range(c["S"]):
        for h in range(c["Hkv"]):
            b = chosen[s, h][chosen[s, h] >= 0].astype(np.int64)
            k, v = _head(c, st, torch.from_numpy(table[s, b]).cuda(), h)
            there = torch.from_numpy(((b[:, None] * bs + np.arange(bs)) < L[s]).reshape(-1)).cuda()
            y = st.q[s, h * G:h * G + G].to(D) @ k[there].T * st.scale
            out[s, h * G:h * G + G] = torch.softmax(y, -1) @ v[there]
    return [out]
