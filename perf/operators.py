"""The operators around the paged decode step, as cases that can be timed: rotary positions with the KV append,
prompt attention and single-token attention with modified scores, and the page operations of the cache.

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
    c = dict(op=op, Hq=28, Hkv=4, d=128, bs=16, fp8=False, shape=1)
    if op == "rope":
        c.update(S=4, n_lo=1, n_hi=1, h_lo=0, h_hi=100, rotary=128, interleaved=False, theta=1e6, factor=1.0)
    elif op in ("prefill", "decode"):
        c.update(S=4, n_lo=1, n_hi=1, h_lo=0, h_hi=100, cap=0.0, bias=False, window=0, doc=0, prefix=0)
    else:
        c.update(S=8, group=8, h_lo=1, h_hi=100)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of a 7B-shaped rollout batch: 256 sequences, one new token each
        _case("rope", name="rope decode 256x1", S=256, h_lo=512, h_hi=8703),
        # a batch of prompts on its way into the cache: interleaved pairs, half of the head, scaled for a long context
        _case("rope", name="rope prompts interleaved", S=12, n_lo=700, n_hi=2100, h_hi=0, Hq=40, Hkv=8, rotary=64,
              interleaved=True, theta=5e5, factor=8.0),
        # a small ragged step over an fp8 cache, far positions
        _case("rope", name="rope fp8 small", S=5, n_lo=1, n_hi=90, h_lo=1000, h_hi=60000, Hq=4, Hkv=1, d=64, rotary=64, fp8=True),
        # the smallest prompts: a few short questions
        _case("prefill", name="prefill tiny", S=4, n_lo=1, n_hi=256, h_hi=0, Hq=4, Hkv=1, d=64, cap=30.0, bias=True),
        # a batch of ordinary ragged prompts, scores capped
        _case("prefill", name="prefill prompts capped", S=16, n_lo=200, n_hi=2048, h_hi=0, cap=50.0),
        # one long prompt, causal
        _case("prefill", name="prefill long causal", S=1, n_lo=8191, n_hi=8191, h_hi=0),
        # chunks of prompts over a long cached history: bidirectional prefix, documents, distance bias
        _case("prefill", name="prefill chunk masked", S=3, n_lo=300, n_hi=600, h_lo=9000, h_hi=16000, Hq=64, Hkv=8, bs=64,
              bias=True, doc=5000, prefix=9200),
        # a handful of short sequences, one new token each
        _case("decode", name="decode tiny capped", S=4, h_hi=255, Hq=4, Hkv=1, d=64, cap=30.0),
        # the 7B-shaped rollout step with capped scores and a distance bias
        _case("decode", name="decode 256 capped biased", S=256, h_lo=512, h_hi=4600, cap=50.0, bias=True),
        # long contexts over an fp8 cache, a sliding window
        _case("decode", name="decode fp8 window", S=48, h_lo=1000, h_hi=32767, Hq=64, Hkv=8, bs=32, fp8=True, window=4096),
        # prompts forked into groups of eight samples
        _case("fork", name="fork 64 prompts x8", S=64, group=8, h_lo=300, h_hi=1500),
        # finished samples freed, the pool compacted
        _case("recycle", name="recycle 384 samples", S=384, h_lo=100, h_hi=1800),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "prefill", "prefill", "prefill", "decode", "decode", "decode", "fork", "recycle"])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16])
    d = rng.choice([64, 128, 128])
    kw = dict(Hkv=Hkv, Hq=Hkv * G, d=d, bs=rng.choice([16, 32, 64]), shape=rng.randrange(1 << 20))
    if op == "rope":
        kw.update(S=_log(rng, 1, 300), h_lo=0, h_hi=_log(rng, 1, 100000) if rng.random() < 0.3 else _log(rng, 1, 3000),
                  interleaved=rng.random() < 0.5, theta=rng.choice([1e4, 5e5, 1e6]), factor=rng.choice([1.0, 4.0, 32.0]),
                  rotary=rng.choice([16, 32, 48, 64] + ([96, 112, 128] if d == 128 else [])), fp8=rng.random() < 0.4)
        if kw["h_hi"] > 3000:
            kw["S"] = min(kw["S"], 12)
        top = max(1, min(2000, 12000 // kw["S"]))
        kw.update(n_lo=1, n_hi=1 if rng.random() < 0.3 else _log(rng, 1, top))
    elif op == "prefill":
        kw["Hq"] = Hkv * (G if Hkv * G <= 32 else max(1, 32 // Hkv))
        n = _log(rng, 1, 3000)
        h = 0 if rng.random() < 0.5 else _log(rng, 1, 6000)
        S = max(1, min(_log(rng, 1, 40), int(6e7 / (n * (n + h) * max(1, kw["Hq"] / 8)))))
        kw.update(S=S, n_lo=max(1, n // 8), n_hi=n, h_lo=h // 4, h_hi=h, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                  bias=rng.random() < 0.4, window=rng.choice([0, 0, _log(rng, 1, 2000)]),
                  doc=rng.choice([0, 0, _log(rng, 1, 2000)]), prefix=rng.choice([0, 0, _log(rng, 1, 3000)]))
    elif op == "decode":
        h = _log(rng, 1, 20000)
        S = max(1, min(_log(rng, 1, 400), int(1.5e6 / (h * max(1, Hkv / 2)))))
        kw.update(S=S, h_lo=h // 6, h_hi=h, cap=rng.choice([0.0, 20.0, 50.0]), bias=rng.random() < 0.5,
                  window=rng.choice([0, 0, _log(rng, 1, 9000)]), doc=rng.choice([0, 0, _log(rng, 1, 9000)]),
                  fp8=rng.random() < 0.4)
    elif op == "fork":
        kw.update(S=_log(rng, 1, 80), group=rng.choice([1, 2, 4, 7, 8, 16]), h_lo=1, h_hi=_log(rng, 2, 1500))
    else:
        kw.update(S=_log(rng, 2, 400), h_lo=1, h_hi=_log(rng, 2, 1500))
    return _case(op, **kw)


def _shape(c):
    """New tokens and context lengths of the case's sequences (the case alone decides them)."""
    r = np.random.default_rng(c["shape"])
    n = r.integers(c["n_lo"], c["n_hi"] + 1, c["S"]) if "n_lo" in c else np.zeros(c["S"], np.int64)
    lo = min(c.get("h_lo", 0), c["h_hi"])
    return n.astype(np.int64), (r.integers(lo, c["h_hi"] + 1, c["S"]) + n).astype(np.int64)


def _interval(c, n, L):
    """First and one-past-last visible key of every new token, sequence after sequence."""
    s = np.repeat(np.arange(len(n)), n)
    j = np.arange(n.sum()) - np.repeat(np.cumsum(n) - n, n)
    pos = L[s] - n[s] + j
    lo = np.zeros_like(pos)
    if c["window"]:
        lo = np.maximum(lo, pos - c["window"] + 1)
    if c["doc"]:
        lo = np.maximum(lo, pos // c["doc"] * c["doc"])
    hi = np.minimum(L[s], np.maximum(pos + 1, c["prefix"]))
    return s, lo, hi


def work(c):
    n, L = _shape(c)
    kv = 2 * c["Hkv"] * c["d"] * (1 if c["fp8"] else 2)
    if c["op"] == "rope":
        N = int(n.sum())
        rows = c["Hq"] + c["Hkv"]
        return {"bytes": N * c["d"] * 2 * (2 * c["Hq"] + 2 * c["Hkv"]) + N * kv, "flops": 3 * N * rows * c["rotary"]}
    if c["op"] in ("prefill", "decode"):
        s, lo, hi = _interval(c, n, L)
        first, last = L.copy(), np.zeros_like(L)
        np.minimum.at(first, s, lo)
        np.maximum.at(last, s, hi)
        keys = int(np.maximum(0, last - first).sum())
        return {"bytes": keys * kv + int(n.sum()) * c["Hq"] * c["d"] * 4,
                "flops": 4 * c["d"] * c["Hq"] * int(np.maximum(0, hi - lo).sum())}
    page = 2 * c["Hkv"] * c["bs"] * c["d"] * 2
    pages = -(-L // c["bs"])
    if c["op"] == "fork":
        return {"bytes": c["group"] * int((L % c["bs"] != 0).sum() * 2 * page + 16 * pages.sum()), "flops": 0}
    live = int(pages[1::2].sum())
    total = int(pages.sum())
    perm = np.random.default_rng(c["shape"] + 1).permutation(total)   # the table's pages, sequence after sequence
    first = np.cumsum(pages) - pages
    keep = np.concatenate([perm[first[i]:first[i] + pages[i]] for i in range(1, c["S"], 2)])
    return {"bytes": int((keep >= live).sum()) * 2 * page + 8 * total, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------
def _i32(x, dev="cuda"):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)


def prepare(c, seed):
    from types import SimpleNamespace
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = _shape(c)
    S, Hq, Hkv, d, bs = c["S"], c["Hq"], c["Hkv"], c["d"], c["bs"]
    pages = -(-L // bs)
    total = int(pages.sum())
    paged = c["op"] in ("fork", "recycle")
    if paged:
        perm = np.random.default_rng(c["shape"] + 1).permutation(total)
    else:
        perm = np.random.default_rng(seed).permutation(total)
    NB = total + (S * c["group"] if c["op"] == "fork" else 0) + 3
    rows = S * (c["group"] + 1) if c["op"] == "fork" else S
    MB = max(1, int(pages.max()))
    table = np.full((rows, MB), -1, np.int32)
    mask = np.arange(MB)[None, :] < pages[:, None]
    table[:S][mask] = perm
    st = SimpleNamespace(c=c, scale=1.0 / math.sqrt(d))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", dtype=BF16, generator=g)

    st.k_cache, st.v_cache = normal(NB, Hkv, bs, d), normal(NB, Hkv, bs, d)
    if c["fp8"]:
        st.k_scale = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
        st.v_scale = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
        st.k_cache = (st.k_cache.float() / st.k_scale.view(1, -1, 1, 1)).to(F8).view(torch.uint8)
        st.v_cache = (st.v_cache.float() / st.v_scale.view(1, -1, 1, 1)).to(F8).view(torch.uint8)
        st.v_cache = st.v_cache.transpose(2, 3).contiguous()
    if paged:
        # the bookkeeping of the pool in one buffer, so that a pass can start from the same books with one copy
        ref = np.zeros(NB, np.int32)
        ref[perm] = 1
        free = np.full(NB, -1, np.int32)
        unused = np.flatnonzero(ref == 0)[::-1]
        free[:len(unused)] = unused
        lens = np.zeros(rows, np.int32)
        lens[:S] = L
        books = np.concatenate([table.reshape(-1), lens, ref, free, [len(unused)]])
        st.books0 = _i32(books)
        st.books = st.books0.clone()
        st.table, st.lens, st.ref, st.free, st.count = (
            x.view(rows, MB) if i == 0 else x
            for i, x in enumerate(torch.split(st.books, [rows * MB, rows, NB, NB, 1])))
        if c["op"] == "fork":
            order = np.random.default_rng(seed).permutation(S * c["group"])
            st.parents, st.children = _i32(np.repeat(np.arange(S), c["group"])[order]), _i32(S + order)
            st.src, st.dst = (torch.empty(S * c["group"], dtype=torch.int32, device="cuda") for _ in range(2))
        else:
            st.finished = _i32(np.random.default_rng(seed).permutation(np.arange(0, S, 2)))
            st.src, st.dst = (torch.empty(NB // 2, dtype=torch.int32, device="cuda") for _ in range(2))
        st.books_ws = torch.zeros(16 * NB + 32768, dtype=torch.uint8, device="cuda")
        return st
    N = int(n.sum())
    st.table, st.lens, st.lens_host = _i32(table), _i32(L), L.astype(np.int32)
    st.cu = _i32(np.concatenate([[0], np.cumsum(n)]))
    st.n_max = int(n.max())
    st.one = bool((n == 1).all())
    if c["op"] == "rope":
        # q, k and v of a token side by side, as a fused projection leaves them
        qkv = normal(N, (Hq + 2 * Hkv), d)
        st.q, st.k, st.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st.q_out = torch.empty(N, Hq, d, device="cuda", dtype=BF16)
        f = c["theta"] ** (-np.arange(0, c["rotary"], 2) / c["rotary"])
        if c["factor"] != 1.0:   # long wavelengths stretched, short ones kept
            f = np.where(2 * math.pi / f > 8192, f / c["factor"], f)
        st.inv_freq = torch.from_numpy(f.astype(np.float32)).cuda()
        st.magnitude = 0.1 * math.log(c["factor"]) + 1.0
        return st
    st.q = normal(N, Hq, d)
    st.out = torch.zeros_like(st.q)
    st.slopes = (2.0 ** (-8.0 * (torch.arange(Hq, device="cuda") + 1) / Hq)).float() if c["bias"] else None
    _, lo, _ = _interval(dict(c, window=0), n, L)
    st.begin_host = lo.astype(np.int32)
    st.begin = _i32(lo) if c["doc"] else None
    st.prefix = torch.full((S,), c["prefix"], dtype=torch.int32, device="cuda") if c["prefix"] else None
    size = (16 * S + 8 * N + (64 << 20)) if c["op"] == "decode" else (1 << 20) + 64 * (N + S) * Hkv
    st.ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------------------------------------------
def _tokens(st):
    """Sequence and position of every new token."""
    N = st.q.shape[0]
    cu = st.cu.long()
    t = torch.arange(N, device="cuda")
    s = torch.searchsorted(cu, t, right=True) - 1
    n = cu[s + 1] - cu[s]
    return s, st.lens.long()[s] - n + (t - cu[s])


def _rotate(x, cos, sin, c):
    r = c["rotary"]
    x = x.float()
    a, rest = x[..., :r], x[..., r:]
    if c["interleaved"]:
        u, v = a[..., 0::2], a[..., 1::2]
        y = torch.stack((u * cos - v * sin, v * cos + u * sin), -1).flatten(-2)
    else:
        u, v = a[..., :r // 2], a[..., r // 2:]
        y = torch.cat((u * cos - v * sin, v * cos + u * sin), -1)
    return torch.cat((y, rest), -1)


def _plain_rope(st):
    c = st.c
    s, pos = _tokens(st)
    angle = pos.double()[:, None] * st.inv_freq.double()
    cos, sin = (angle.cos() * st.magnitude).float()[:, None], (angle.sin() * st.magnitude).float()[:, None]
    q = _rotate(st.q, cos, sin, c).to(BF16)
    k = _rotate(st.k, cos, sin, c)
    page, slot = st.table[s, pos // c["bs"]].long(), pos % c["bs"]
    if c["fp8"]:
        ks, vs = st.k_scale.view(1, -1, 1), st.v_scale.view(1, -1, 1)
        st.k_cache.view(F8)[page, :, slot] = (k / ks).clamp(-448, 448).to(F8)
        st.v_cache.view(F8)[page, :, :, slot] = (st.v.float() / vs).clamp(-448, 448).to(F8)
        return [q, st.k_cache.view(F8), st.v_cache.view(F8)]
    st.k_cache[page, :, slot] = k.to(BF16)
    st.v_cache[page, :, slot] = st.v
    return [q, st.k_cache, st.v_cache]


def _gathered(st):
    """K and V of every sequence, in 32 bits: [S, Hkv, keys, d]."""
    c = st.c
    at = st.table.clamp(min=0).long()
    if c["fp8"]:
        k = st.k_cache.view(F8)[at].float() * st.k_scale.view(1, 1, -1, 1, 1)
        v = st.v_cache.view(F8)[at].float().transpose(3, 4) * st.v_scale.view(1, 1, -1, 1, 1)
    else:
        k, v = st.k_cache[at].float(), st.v_cache[at].float()
    S, P = at.shape
    return (x.transpose(1, 2).reshape(S, c["Hkv"], P * c["bs"], c["d"]) for x in (k, v))


def _plain_attention(st):
    c = st.c
    S, Hq, Hkv, d, n = c["S"], c["Hq"], c["Hkv"], c["d"], st.n_max
    G = Hq // Hkv
    s, pos = _tokens(st)
    j = torch.arange(st.q.shape[0], device="cuda") - st.cu.long()[s]
    q = torch.zeros(S, n, Hq, d, device="cuda")
    q[s, j] = st.q.float()
    k, v = _gathered(st)
    x = (q * st.scale).view(S, n, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * n, d)
    x = torch.matmul(x, k.transpose(2, 3)).view(S, Hkv, G, n, -1)
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    t = torch.arange(k.shape[2], device="cuda")
    p = torch.zeros(S, n, dtype=torch.long, device="cuda")
    p[s, j] = pos
    if st.slopes is not None:
        x = x - st.slopes.view(1, Hkv, G, 1, 1) * (p[:, None, None, :, None] - t).abs()
    lo = torch.zeros_like(p)
    if c["window"]:
        lo = (p - c["window"] + 1).clamp(min=0)
    if st.begin is not None:
        b = torch.zeros_like(p)
        b[s, j] = st.begin.long()
        lo = torch.maximum(lo, b)
    hi = p + 1
    if st.prefix is not None:
        hi = torch.maximum(hi, st.prefix.long()[:, None])
    hi = torch.minimum(hi, st.lens.long()[:, None])
    seen = (t >= lo[..., None]) & (t < hi[..., None])
    x = torch.where(seen[:, None, None], x, float("-inf"))
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == float("-inf"), 0.0, m))
    total = e.sum(-1, keepdim=True)
    e = e / torch.where(total > 0, total, 1.0)
    o = torch.matmul(e.view(S, Hkv, G * n, -1), v).view(S, Hkv, G, n, d).permute(0, 3, 1, 2, 4).reshape(S, n, Hq, d)
    return [o[s, j].to(BF16)]


def _plain_fork(st):
    bs = st.c["bs"]
    p, ch = st.parents.long(), st.children.long()
    L = st.lens[p]
    cols = torch.arange(st.table.shape[1], device="cuda")
    rows = st.table[p]
    whole = cols < (L // bs)[:, None]
    tail = L % bs != 0
    rank = torch.cumsum(tail, 0) - 1
    top = st.count.long() - 1
    page = torch.where(tail, st.free[(top - rank).clamp(min=0)], -1)
    at = torch.where(tail, rank, torch.cumsum(~tail, 0) - 1 + tail.sum())
    st.src[at] = torch.where(tail, rows.gather(1, (L // bs).long().clamp(max=len(cols) - 1)[:, None])[:, 0], -1)
    st.dst[at] = page
    st.ref.index_add_(0, rows.clamp(min=0).view(-1).long(), whole.view(-1).int())
    st.ref.index_add_(0, page.clamp(min=0).long(), tail.int())
    is_tail = (cols == (L // bs)[:, None]) & tail[:, None]
    st.table[ch] = torch.where(whole, rows, torch.where(is_tail, page[:, None], -1))
    st.lens[ch] = L
    st.count -= tail.sum().int()
    st.free[:] = torch.where(torch.arange(len(st.free), device="cuda") < st.count, st.free, -1)
    _plain_copy(st)
    return [st.books, st.src, st.dst, st.k_cache, st.v_cache]


def _plain_copy(st):
    # a pair of -1 stands for no copy: it goes from the last page to itself, which nothing here moves
    n = st.k_cache.shape[0] - 1
    src, dst = torch.where(st.src < 0, n, st.src).long(), torch.where(st.dst < 0, n, st.dst).long()
    st.k_cache[dst] = st.k_cache[src]
    st.v_cache[dst] = st.v_cache[src]


def _rebuild(st):
    """The free list: pages without references, the lowest id last; -1 past the end."""
    free = st.ref == 0
    n = free.sum()
    ids = torch.arange(len(free), device="cuda")
    at = torch.where(free, n - torch.cumsum(free, 0), n + torch.cumsum(~free, 0) - 1)
    st.free[at] = torch.where(free, ids, -1).int()
    st.count[0] = n


def _plain_recycle(st):
    bs, cols = st.c["bs"], torch.arange(st.table.shape[1], device="cuda")
    f = st.finished.long()
    mine = cols < (-(-st.lens[f] // bs))[:, None]
    st.ref.index_add_(0, st.table[f].clamp(min=0).view(-1).long(), -mine.view(-1).int())
    st.table[f] = -1
    st.lens[f] = 0
    # compaction: the live pages past the number of live pages move, in ascending order, into the holes below it
    live = st.ref > 0
    n = live.sum()
    ids = torch.arange(len(live), device="cuda")
    hole, mover = ~live & (ids < n), live & (ids >= n)
    st.src.fill_(-1)
    st.dst.fill_(-1)
    k = len(st.src)
    padded = torch.cat((st.src, st.src[:1])), torch.cat((st.dst, st.dst[:1]))
    for_mover = torch.where(mover, torch.cumsum(mover, 0) - 1, k)
    padded[0][for_mover] = torch.where(mover, ids, -1).int()
    padded[1][torch.where(hole, torch.cumsum(hole, 0) - 1, k)] = torch.where(hole, ids, -1).int()
    st.src[:] = padded[0][:k]
    st.dst[:] = padded[1][:k]
    to = torch.where(mover, padded[1][for_mover].long(), ids)
    used = cols < (-(-st.lens // bs))[:, None]
    st.table[:] = torch.where(used, to[st.table.clamp(min=0).long()].int(), st.table)
    ref = torch.zeros_like(st.ref)
    st.ref[:] = ref.index_add_(0, to, st.ref)
    _rebuild(st)
    _plain_copy(st)
    return [st.books, st.src, st.dst, st.k_cache, st.v_cache]


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------
def run(st):
    c = st.c
    if c["op"] in ("fork", "recycle"):
        st.books.copy_(st.books0)   # every pass starts from the same books
    if own:
        return _own(st)
    return {"rope": _plain_rope, "prefill": _plain_attention, "decode": _plain_attention, "fork": _plain_fork,
            "recycle": _plain_recycle}[c["op"]](st)


def _own(st):
    from paper_2607_09207_b200 import pdattn
    c = st.c
    if c["op"] == "rope":
        kw = dict(cu_tokens=None if st.one else st.cu, rotary_dim=c["rotary"], interleaved=c["interleaved"],
                  magnitude=st.magnitude)
        if c["fp8"]:
            pdattn.rope_append_fp8(st.q, st.k, st.v, st.q_out, st.k_cache, st.v_cache, st.k_scale, st.v_scale, st.table,
                                   st.lens, st.inv_freq, **kw)
            return [st.q_out, st.k_cache.view(F8), st.v_cache.view(F8)]
        pdattn.rope_append(st.q, st.k, st.v, st.q_out, st.k_cache, st.v_cache, st.table, st.lens, st.inv_freq, **kw)
        return [st.q_out, st.k_cache, st.v_cache]
    if c["op"] in ("prefill", "decode"):
        score = pdattn.Score(logit_cap=c["cap"], bias_slopes=st.slopes, window=c["window"], key_begin=st.begin,
                             prefix_lens=st.prefix, key_begin_host=st.begin_host if c["doc"] else None)
        if c["op"] == "prefill":
            pdattn.prefill(st.q, st.k_cache, st.v_cache, st.table, st.lens, st.cu, st.scale, st.out, st.ws, score=score)
        elif c["fp8"]:
            pdattn.decode_scored_fp8(st.q, st.k_cache, st.v_cache, st.k_scale, st.v_scale, st.table, st.lens, st.scale,
                                     st.out, st.ws, score, context_lens_host=st.lens_host)
        else:
            pdattn.decode_scored(st.q, st.k_cache, st.v_cache, st.table, st.lens, st.scale, st.out, st.ws, score,
                                 context_lens_host=st.lens_host)
        return [st.out]
    pool = pdattn.PagePool(st.ref, st.free, st.count)
    if c["op"] == "fork":
        pdattn.pages_fork(pool, st.table, st.lens, st.parents, st.children, st.src, st.dst, c["bs"], st.books_ws)
    else:
        pdattn.pages_free(pool, st.table, st.lens, st.finished, c["bs"], st.books_ws)
        pdattn.pages_compact(pool, st.table, st.lens, st.src, st.dst, c["bs"], st.books_ws)
    pdattn.pages_copy(st.k_cache, st.v_cache, st.src, st.dst)
    return [st.books, st.src, st.dst, st.k_cache, st.v_cache]


# ---------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(c, seed):
    st = prepare(c, seed)
    n, L = _shape(c)
    if c["op"] in ("fork", "recycle"):
        return _exact_pages(c, st, L)
    bs, G, D = c["bs"], c["Hq"] // c["Hkv"], torch.float64
    table = st.table.cpu().numpy().astype(np.int64)
    cu = np.concatenate([[0], np.cumsum(n)])
    if c["op"] == "rope":
        R = c["rotary"]
        f = st.inv_freq.to(D)
        q_out = torch.empty(st.q.shape, dtype=D, device="cuda")
        if c["fp8"]:
            kc, vc = st.k_cache.view(F8).to(D), st.v_cache.view(F8).to(D)
            ks, vs = st.k_scale.to(D)[:, None], st.v_scale.to(D)[:, None]
        else:
            kc, vc = st.k_cache.to(D), st.v_cache.to(D)
            ks = vs = 1.0
        even, odd = (np.arange(0, R, 2), np.arange(1, R, 2)) if c["interleaved"] else (np.arange(R // 2), np.arange(R // 2, R))
        for s in range(c["S"]):
            span = slice(int(cu[s]), int(cu[s + 1]))
            pos = np.arange(L[s] - n[s], L[s])
            z = torch.polar(torch.full((len(pos), R // 2), st.magnitude, dtype=D, device="cuda"),
                            torch.from_numpy(pos).cuda().to(D)[:, None] * f)[:, None]

            def turned(x):
                x = x.to(D).clone()
                w = torch.complex(x[..., even], x[..., odd]) * z
                x[..., even], x[..., odd] = w.real, w.imag
                return x
            q_out[span] = turned(st.q[span])
            page, slot = torch.from_numpy(table[s, pos // bs]).cuda(), torch.from_numpy(pos % bs).cuda()
            kc[page, :, slot] = turned(st.k[span]) / ks
            if c["fp8"]:
                vc[page, :, :, slot] = st.v[span].to(D) / vs
            else:
                vc[page, :, slot] = st.v[span].to(D)
        return [q_out, kc, vc]
    out = torch.zeros(st.q.shape, dtype=D, device="cuda")
    _, lo, hi = _interval(c, n, L)
    for s in range(c["S"]):
        span = slice(int(cu[s]), int(cu[s + 1]))
        at = torch.from_numpy(table[s, :-(-int(L[s]) // bs)]).cuda()
        pos = torch.arange(int(L[s] - n[s]), int(L[s]), device="cuda")
        t = torch.arange(int(L[s]), device="cuda")
        dist = (pos[:, None] - t).abs().to(D)
        a, b = (torch.from_numpy(x[span]).cuda()[:, None] for x in (lo, hi))
        hidden = ~((t >= a) & (t < b))
        for h in range(c["Hkv"]):
            if c["fp8"]:
                k = st.k_cache[at, h].view(F8).to(D).reshape(-1, c["d"])[:int(L[s])] * st.k_scale[h].to(D)
                v = st.v_cache[at, h].view(F8).to(D).transpose(1, 2).reshape(-1, c["d"])[:int(L[s])] * st.v_scale[h].to(D)
            else:
                k, v = (x[at, h].to(D).reshape(-1, c["d"])[:int(L[s])] for x in (st.k_cache, st.v_cache))
            for i in range(h * G, h * G + G):
                y = st.q[span, i].to(D) @ k.T * st.scale
                if c["cap"]:
                    y = c["cap"] * torch.tanh(y / c["cap"])
                if st.slopes is not None:
                    y -= st.slopes[i].to(D) * dist
                y.masked_fill_(hidden, -math.inf)
                out[span, i] = torch.nan_to_num(torch.softmax(y, -1), nan=0.0) @ v
    return [out]


def _exact_pages(c, st, L):
    bs = c["bs"]
    table, lens, ref = st.table.cpu().numpy(), st.lens.cpu().numpy(), st.ref.cpu().numpy()
    src, dst = np.full(len(st.src), -1, np.int32), np.full(len(st.dst), -1, np.int32)
    pairs = []
    if c["op"] == "fork":
        unused = sorted(np.flatnonzero(ref == 0).tolist())
        for p, ch in zip(st.parents.tolist(), st.children.tolist()):
            whole, tail = divmod(int(lens[p]), bs)
            table[ch] = -1
            table[ch, :whole] = table[p, :whole]
            ref[table[p, :whole]] += 1
            if tail:
                page = unused.pop(0)
                pairs.append((int(table[p, whole]), page))
                table[ch, whole] = page
                ref[page] = 1
            lens[ch] = lens[p]
    else:
        for s in st.finished.tolist():
            ref[table[s, :-(-int(lens[s]) // bs)]] -= 1
            table[s], lens[s] = -1, 0
        live = int((ref > 0).sum())
        pairs = list(zip((live + np.flatnonzero(ref[live:] > 0)).tolist(), np.flatnonzero(ref[:live] == 0).tolist()))
        move = dict(pairs)
        for s in range(len(lens)):
            for b in range(-(-int(lens[s]) // bs)):
                table[s, b] = move.get(int(table[s, b]), int(table[s, b]))
        for a, b in pairs:
            ref[a], ref[b] = 0, ref[a]
        unused = np.flatnonzero(ref == 0).tolist()
    for i, (a, b) in enumerate(pairs):
        src[i], dst[i] = a, b
    k, v = st.k_cache.double(), st.v_cache.double()
    if pairs:
        a, b = (torch.tensor(x, device="cuda") for x in zip(*pairs))
        k[b], v[b] = k[a], v[a]
    free = np.full(len(ref), -1, np.int32)
    free[:len(unused)] = unused[::-1]
    books = np.concatenate([table.reshape(-1), lens, ref, free, [len(unused)]])
    return [books.astype(np.int32), src, dst, k, v]
