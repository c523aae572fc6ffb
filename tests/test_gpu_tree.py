"""Attention for trees of drafted tokens, the accepted path, and what goes with them, against their definitions."""
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


def trees(n, seed=0):
    """Masks of random trees: a token continues any earlier one, or none."""
    r = np.random.default_rng(seed)
    out = []
    for x in n:
        m = []
        for j in range(x):
            p = int(r.integers(-1, j)) if j else -1
            m.append((m[p] if p >= 0 else 0) | 1 << j)
        out += m
    return out


class Case:
    """Sequences of L tokens, the last n of them drafted; slots that no sequence owns hold NaN."""

    def __init__(self, n, L, Hq, Hkv, d, bs, seed=0, masks=None, fp8=False, nhd=False, MB=None):
        self.n, self.L, self.bs, self.fp8 = np.asarray(n), np.asarray(L), bs, fp8
        g = torch.Generator(device="cuda").manual_seed(seed)
        S, N = len(n), int(self.n.sum())
        pages = -(-self.L // bs)
        NB = int(pages.sum()) + 2
        perm = np.random.default_rng(seed).permutation(NB)
        self.tab = np.full((S, MB or max(1, int(pages.max()))), -1, np.int32)
        at = 0
        shape = (NB, bs, Hkv, d) if nhd else (NB, Hkv, bs, d)
        self.k, self.v = (torch.randn(*shape, device="cuda", dtype=BF16, generator=g) for _ in range(2))
        if nhd:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        dead = torch.ones(NB, bs, dtype=torch.bool)
        for s in range(S):
            own = perm[at:at + pages[s]]
            at += pages[s]
            m = min(len(own), self.tab.shape[1])
            self.tab[s, :m] = own[:m]
            for b, p in enumerate(own):
                dead[p, :max(0, min(bs, int(self.L[s]) - b * bs))] = False
        for x in (self.k, self.v):
            x.masked_fill_(dead.cuda()[:, None, :, None].expand_as(x), math.nan)
        self.q = torch.randn(N, Hq, d, device="cuda", dtype=BF16, generator=g) * 2
        self.masks = trees(self.n, seed) if masks is None else masks
        self.cu = np.concatenate([[0], np.cumsum(self.n)])
        self.scale = 1.0 / math.sqrt(d)
        if fp8:
            self.ks = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
            self.vs = torch.rand(Hkv, device="cuda", generator=g) * 0.02 + 0.02
            self.k = (self.k.float() / self.ks.view(1, -1, 1, 1)).to(F8).view(torch.uint8)
            self.v = (self.v.float() / self.vs.view(1, -1, 1, 1)).to(F8).view(torch.uint8).transpose(2, 3).contiguous()
        self.ws = pdattn.alloc_tree_workspace(Hq, Hkv, d, bs)

    def mask_tensor(self):
        return torch.from_numpy(np.array([m & (2 ** 64 - 1) for m in self.masks], np.uint64).view(np.int64)).cuda()

    def call(self, out, top=None, ws=None, stream=None):
        ws = self.ws if ws is None else ws
        top = int(self.n.max()) if top is None else top
        rest = (self.dev_tab, self.dev_lens, self.dev_cu, self.dev_mask, self.scale, out, ws)
        if self.fp8:
            pdattn.decode_tree_fp8(self.q, self.k, self.v, self.ks, self.vs, *rest, max_tree_tokens=top, stream=stream)
        else:
            pdattn.decode_tree(self.q, self.k, self.v, *rest, max_tree_tokens=top, stream=stream)

    def upload(self):
        self.dev_tab, self.dev_lens, self.dev_cu, self.dev_mask = i32(self.tab), i32(self.L), i32(self.cu), self.mask_tensor()
        return self

    def run(self, top=None, expect=pdattn.OK):
        out = torch.full_like(self.q, 7.0)
        self.upload().call(out, top)
        assert pdattn.check(self.ws) == expect
        return out

    def kv(self):
        if not self.fp8:
            return self.k.double(), self.v.double()
        return (self.k.view(F8).double() * self.ks.double().view(1, -1, 1, 1),
                self.v.view(F8).double().transpose(2, 3) * self.vs.double().view(1, -1, 1, 1))

    def want(self, scale=None):
        """Output and sum of weight times |v|, in 64 bits."""
        N, Hq, d = self.q.shape
        Hkv, NB = self.k.shape[1], self.k.shape[0]
        G, bs = Hq // Hkv, self.bs
        k, v = self.kv()
        out, size = (torch.zeros(N, Hq, d, dtype=torch.double, device="cuda") for _ in range(2))
        for s in range(len(self.n)):
            n, L = int(self.n[s]), int(self.L[s])
            keys = min(L, self.tab.shape[1] * bs)
            if n == 0 or keys == 0:
                continue
            pg = torch.from_numpy(self.tab[s, :-(-keys // bs)].astype(np.int64)).cuda()
            ok = (pg >= 0) & (pg < NB)
            pg = torch.where(ok, pg, 0)
            vis = np.zeros((n, keys), bool)
            for j in range(n):
                if L - n + j < 0:
                    continue
                vis[j, :max(0, min(keys, L - n))] = True
                for i in range(n):
                    if self.masks[self.cu[s] + j] >> i & 1 and 0 <= L - n + i < keys:
                        vis[j, L - n + i] = True
            vis = torch.from_numpy(vis).cuda() & ok.repeat_interleave(bs)[None, :keys]
            sp = slice(int(self.cu[s]), int(self.cu[s + 1]))
            for h in range(Hkv):
                kk, vv = (x[pg, h].reshape(-1, d)[:keys] for x in (k, v))
                x = torch.einsum("jgd,td->gjt", self.q[sp, h * G:h * G + G].double(), kk) * (self.scale if scale is None else scale)
                p = torch.nan_to_num(torch.softmax(x.masked_fill(~vis, -math.inf), -1), nan=0.0)
                vv = torch.where(vis.any(0)[:, None], vv, 0.0)
                out[sp, h * G:h * G + G] = torch.einsum("gjt,td->jgd", p, vv)
                size[sp, h * G:h * G + G] = torch.einsum("gjt,td->jgd", p, vv.abs())
        return out.cpu().numpy(), size.cpu().numpy()


def close(got, want, size, fp8=False):
    # the result is rounded once (2^-8 of it); the weights are rounded once (bf16 2^-8 of each, fp16 2^-11; over codes q is off by
    # 2^-17.8 of a row's largest, 2^-13 of the weight for sums of |k| up to a few hundred); scores and sums are fp32 with exponentials good to 2^-22 (below 2^-12 of sum p |v| for scores up to a few hundred)
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    err, tol = abs(got - want), 2.0 ** -8 * abs(want) + ((2.0 ** -11 if fp8 else 2.0 ** -8) + 2.0 ** -12) * size + 1e-30
    assert (err <= tol).all(), (err / tol).max()


SHAPES = [(28, 4, 128, 16), (4, 1, 64, 16), (16, 1, 128, 32), (12, 1, 64, 64), (8, 8, 128, 64), (6, 2, 64, 32), (10, 2, 128, 16)]


@pytest.mark.parametrize("Hq,Hkv,d,bs", SHAPES)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("top", [8, 64])
def test_trees(Hq, Hkv, d, bs, fp8, top):
    """Trees of at most 8 (one row tile) and of up to 64 tokens (up to eight), without a history and over one to fifteen key tiles."""
    n = np.array([1, 2, 8, 7, 3, 0, 5, 8, 1, 6, 4, 8]) if top == 8 else np.array([64, 1, 63, 33, 17, 0, 64, 40, 5, 64, 18, 36])
    L = n + np.array([0, 0, 0, 120, 125, 50, 128, 250, 383, 900, 1800, 127])
    c = Case(n, L, Hq, Hkv, d, bs, seed=Hq, fp8=fp8)
    close(c.run(), *c.want(), fp8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,bs", [(128, 16), (64, 64), (128, 32), (64, 32)])
@pytest.mark.parametrize("n", [[3, 5, 8], [64, 20, 40]])
def test_long_contexts_are_cut(fp8, d, bs, n):
    """Few units over many key tiles: every CTA has pieces of cut units, in both forms."""
    n = np.array(n)
    c = Case(n, n + np.array([9000, 30000, 127]), 14, 2, d, bs, seed=5, fp8=fp8)
    a = c.run()
    close(a, *c.want(), fp8)
    assert torch.equal(c.run(), a)


@pytest.mark.parametrize("fp8", [False, True])
def test_one_token_one_key(fp8):
    for L in (1, 2, 127, 128, 129, 16, 17):
        c = Case([1], [L], 4, 2, 64, 16, fp8=fp8)
        close(c.run(), *c.want(), fp8)


@pytest.mark.parametrize("fp8", [False, True])
def test_many_short_sequences(fp8):
    r = np.random.default_rng(0)
    n = r.integers(0, 7, 700)
    c = Case(n, n + r.integers(0, 300, 700), 8, 2, 128, 16, seed=2, fp8=fp8)
    close(c.run(), *c.want(), fp8)


@pytest.mark.parametrize("d,Hq", [(64, 24), (128, 56)])
@pytest.mark.parametrize("top", [16, 64])
def test_short_sequences_in_numbers(d, Hq, top):
    """Every CTA has several units of one or two key tiles: queries come and go faster than their weights."""
    rng = np.random.default_rng(d + top)
    n = rng.integers(1, top + 1, 200)
    for fp8 in (True, False):
        c = Case(n, n + rng.integers(0, 100, 200), Hq, 8, d, 64, seed=top, fp8=fp8)
        first = c.run(top)
        close(first, *c.want(), fp8)
        for _ in range(20):
            assert torch.equal(c.run(top), first)


def test_lengths_of_every_kind():
    """One long among many short: shares begin and end inside sequences of every length."""
    r = np.random.default_rng(1)
    n = r.integers(1, 17, 150)
    h = r.integers(0, 400, 150)
    h[70], h[71], h[149] = 40000, 5000, 3000
    c = Case(n, n + h, 8, 1, 64, 64, seed=3)
    close(c.run(), *c.want())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_masks_of_every_kind(fp8, d):
    """Any bits: none (an empty row where there is no history), all, later tokens, bits past the tree, a chain."""
    r = np.random.default_rng(4)
    n = np.array([5, 64, 40, 64, 3])
    masks = [0, 0, 1, 31, ~0] + [int(x) for x in r.integers(0, 2 ** 63, 64)] + [(1 << j + 1) - 1 for j in range(40)]
    masks += [~0 << 60 if j % 2 else 0 for j in range(64)] + [1 << 2, ~0, 1 << 63]
    c = Case(n, n + np.array([0, 0, 90, 200, 0]), 8, 2, d, 16, masks=masks, fp8=fp8)
    out = c.run()
    close(out, *c.want(), fp8)
    assert not out[0].any() and not out[1].any() and not out[-1].any()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_chain_is_the_plain_step(fp8):
    """Masks of a chain: pdattn_decode_multi's definition."""
    T, S = 4, 6
    w = W.make_custom([700, 64, 65, 129, 3000, 4], 8, 2, 128, 16, device="cuda:0")
    q = torch.randn(S, T, 8, 128, device="cuda", dtype=BF16)
    one = torch.full((2,), 0.03, device="cuda")
    k8, v8 = W.fp8_caches(w, one, one)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws, wt = pdattn.alloc_multi_workspace(S, 8, 2, 128, 16, T), pdattn.alloc_tree_workspace(8, 2, 128)
    cu, mask = i32(np.arange(S + 1) * T), torch.tensor([1, 3, 7, 15] * S, device="cuda")
    rows = (q.view(S * T, 8, 128), b.view(S * T, 8, 128))
    if fp8:
        pdattn.decode_fp8(q, k8, v8, one, one, w.block_table, w.context_lens, w.scale, a, ws)
        pdattn.decode_tree_fp8(rows[0], k8, v8, one, one, w.block_table, w.context_lens, cu, mask, w.scale, rows[1], wt, max_tree_tokens=T)
    else:
        pdattn.decode_multi(q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, a, ws)
        pdattn.decode_tree(rows[0], w.k_cache, w.v_cache, w.block_table, w.context_lens, cu, mask, w.scale, rows[1], wt, max_tree_tokens=T)
    # both are within 2^-8 of sum p |v| (weights) and 2^-8 of the result (rounding) of the definition; |v| stays below 6
    assert pdattn.check(wt) == pdattn.OK
    assert float((a.float() - b.float()).abs().max()) <= 4 * 2.0 ** -8 * 6


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0, 1e-4])
@pytest.mark.parametrize("fp8", [False, True])
def test_scales(scale, fp8):
    n = np.array([5, 60, 9])
    c = Case(n, n + np.array([300, 140, 0]), 8, 2, 128, 16, fp8=fp8)
    c.scale = scale
    if scale == 3.0:
        c.q.mul_(0.1)
    if fp8:
        c.ks[1] = -c.ks[1]
    close(c.run(), *c.want(), fp8)


def test_other_strides():
    for d, bs in ((128, 16), (64, 32)):
        n = np.array([5, 20])
        c = Case(n, n + np.array([300, 140]), 8, 2, d, bs, nhd=True)
        close(c.run(), *c.want())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n", [[6, 9], [64, 30]])
def test_what_a_token_does_not_see_may_be_anything(fp8, n):
    """NaN and infinities in one branch's K and V: the tokens outside it are as ever; those inside get what is not finite."""
    n = np.array(n)
    masks = [1 << j | 1 for j in range(n[0])] + [1 << j | 1 for j in range(n[1])]      # a root and its children
    c = Case(n, n + np.array([250, 70]), 8, 2, 128, 16, masks=masks, fp8=fp8)
    want = c.want()
    hit = []
    for s, j in ((0, 3), (1, 5), (0, 1)):
        t = int(c.L[s] - n[s] + j)
        p, slot = c.tab[s, t // 16], t % 16
        if fp8:
            c.k[p, 0, slot, 3] = 0x7f
            c.v[p, :, 9, slot] = 0xff
        else:
            c.k[p, 0, slot, 3] = math.inf
            c.v[p, :, slot, 9] = math.nan if j == 3 else -math.inf
        hit.append(int(c.cu[s] + j))
    out = c.run()
    rest = np.setdiff1d(np.arange(int(n.sum())), hit)
    close(out[rest], want[0][rest], want[1][rest], fp8)
    for x in hit:
        assert not out[x, :, 9].isfinite().any()
        assert out[x, 4:, :9].isfinite().all() and out[x, 4:, 10:].isfinite().all()    # (heads of the KV head whose K is whole)
    # in the history, that is seen by all
    c = Case(n, n + np.array([250, 70]), 8, 2, 128, 16, masks=masks, fp8=fp8)
    p = c.tab[0, 3]
    if fp8:
        c.v[p, 1, 9, 2] = 0x7f
    else:
        c.v[p, 1, 2, 9] = math.inf
    out = c.run()
    assert not out[:n[0], 4:, 9].isfinite().any() and out[:n[0], :4].isfinite().all() and out[n[0]:].isfinite().all()


@pytest.mark.parametrize("d,G", [(128, 7), (64, 4), (128, 2), (64, 16)])
@pytest.mark.parametrize("n", [4, 9, 64])
@pytest.mark.parametrize("hist", [200, 9000])
def test_infinities_that_every_token_sees(d, G, n, hist):
    """Of the history's V: an infinity alone gives itself, infinities of both signs or a NaN give NaN, the other channels stay."""
    ns = np.array([n, 1, max(1, n - 1)])
    c = Case(ns, ns + np.array([hist, 70, hist // 2]), G, 1, d, 32, seed=d + G)
    want, size = c.want()
    for s in (0, 2):
        for key, channel, x in [(5, 0, math.inf), (40, 3, -math.inf), (77, d - 1, math.inf), (3, 9, math.inf), (61, 9, -math.inf), (90, 33, math.nan)]:
            c.v[int(c.tab[s, key // 32]), 0, key % 32, channel] = x
        rows = slice(int(c.cu[s]), int(c.cu[s + 1]))
        for channel, x in [(0, math.inf), (3, -math.inf), (d - 1, math.inf), (9, math.nan), (33, math.nan)]:
            want[rows, :, channel] = x
    got = c.run()
    odd = ~np.isfinite(want)
    assert (np.isnan(want[odd]) == np.isnan(got.double().cpu().numpy()[odd])).all()
    assert np.array_equal(np.nan_to_num(want[odd], posinf=1, neginf=-1), np.nan_to_num(got.double().cpu().numpy()[odd], posinf=1, neginf=-1))
    odd = torch.from_numpy(odd).cuda()
    close(torch.where(odd, 0, got), np.where(odd.cpu().numpy(), 0, want), size)


@pytest.mark.parametrize("fp8", [False, True])
def test_bad_pages_and_rows_that_are_too_short(fp8):
    n = np.array([6, 40, 7])
    c = Case(n, n + np.array([500, 700, 900]), 8, 2, 64, 16, fp8=fp8, MB=50)
    out = c.run(expect=pdattn.BAD_PAGE_INDEX)                            # 907 tokens, a row of 800
    close(out, *c.want(), fp8)
    c = Case(n, n + np.array([500, 700, 900]), 8, 2, 64, 16, fp8=fp8)
    c.tab[0, 3], c.tab[0, 30], c.tab[1, 45], c.tab[2, 0] = -5, 1 << 30, c.k.shape[0], -1
    out = c.run(expect=pdattn.BAD_PAGE_INDEX)
    close(out, *c.want(), fp8)
    assert pdattn.check(c.ws) == pdattn.OK


def test_rows_that_are_left_as_they_are():
    """Behind the last sequence, and of a tree with more tokens than announced; a tree longer than its context."""
    n = np.array([5, 9, 3, 4])
    c = Case(n, np.array([100, 60, 3, 2]), 8, 2, 64, 16)
    c.upload()
    more = torch.randn(30, 8, 64, device="cuda", dtype=BF16)
    more[:21] = c.q
    c.q = more
    c.dev_mask = torch.cat((c.dev_mask, torch.zeros(9, dtype=torch.int64, device="cuda")))
    out = torch.full_like(c.q, 7.0)
    c.call(out, top=8)
    assert pdattn.check(c.ws) == pdattn.UNSUPPORTED
    assert (out[5:14] == 7).all() and (out[21:] == 7).all()
    c.q = c.q[:21]
    want, size = c.want()
    keep = np.r_[0:5, 14:21]
    close(out[keep], want[keep], size[keep])
    assert not out[17:19].any()                                          # two tokens of four lie before position 0


def test_results_do_not_depend_on_the_pages_numbers():
    n = np.array([8, 30, 64])
    c = Case(n, n + np.array([5000, 200, 9000]), 8, 2, 128, 16, seed=8)
    a = c.run()
    perm = torch.randperm(c.k.shape[0], device="cuda")
    k, v = torch.empty_like(c.k), torch.empty_like(c.v)
    k[perm], v[perm] = c.k, c.v
    c.k, c.v = k, v
    c.tab = np.where(c.tab >= 0, perm.cpu().numpy()[c.tab.clip(0)], -1)
    assert torch.equal(c.run(), a)


@pytest.mark.parametrize("top", [8, 64])
def test_captured_replayed_and_on_streams_of_their_own(top):
    n = np.array([5, 8, 2]) if top == 8 else np.array([64, 8, 20])
    a = Case(n, n + np.array([3000, 10, 700]), 8, 2, 128, 16, seed=1).upload()
    b = Case(n, n + np.array([100, 2500, 40]), 8, 2, 128, 16, seed=2, fp8=True).upload()
    oa, ob = torch.zeros_like(a.q), torch.zeros_like(b.q)
    a.call(oa, top)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call(oa, top)
    a.q.mul_(-0.5)
    a.L = a.L - 16
    a.dev_lens.sub_(16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        graph.replay()
        b.call(ob, top, stream=side)
    torch.cuda.synchronize()
    close(oa, *a.want())
    close(ob, *b.want(), True)
    assert pdattn.check(a.ws) == pdattn.check(b.ws) == pdattn.OK


def test_wrapper_refuses_what_the_library_cannot_see():
    c = Case([3, 4], [30, 9], 8, 2, 64, 16).upload()
    out = torch.empty_like(c.q)
    good = [c.q, c.k, c.v, c.dev_tab, c.dev_lens, c.dev_cu, c.dev_mask, 0.1, out, c.ws]
    for i, bad in ((0, c.q[:3]), (5, c.dev_cu[:2]), (6, c.dev_mask[:6]), (6, c.dev_mask.int()), (6, c.dev_mask.double()), (8, out[:, :4]),
                   (3, c.dev_tab.long()), (1, c.k.float()), (5, c.dev_cu.cpu())):
        args = list(good)
        args[i] = bad
        with pytest.raises((ValueError, TypeError)):
            pdattn.decode_tree(*args, max_tree_tokens=8)
    for top, what in ((65, pdattn.UNSUPPORTED), (0, pdattn.INVALID_ARG)):
        assert pdattn.decode_tree(*good, max_tree_tokens=top, check=False) == what
    assert pdattn.decode_tree(*good[:9], c.ws[:1 << 20], max_tree_tokens=8, check=False) == pdattn.WORKSPACE_TOO_SMALL


# ---------------------------------------------------------------------------------------------------------------
# The accepted path
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,bs,Hkv", [(128, 16, 4), (64, 32, 1), (64, 64, 3), (128, 64, 2)])
@pytest.mark.parametrize("kind", ["bf16", "nhd", "fp8"])
def test_accepted_paths(d, bs, Hkv, kind):
    n = np.array([64, 1, 5, 0, 33, 64, 7, 20, 3])
    L = n + np.array([0, 0, 13, 5, 100, bs - 1, 3 * bs, 2, 40])
    paths = [list(range(64)), [0], [1, 2, 4], [], [0, 3, 30, 32], [63], list(range(1, 7)), list(range(0, 20, 2)), []]
    c = Case(n, L, 2 * Hkv, Hkv, d, bs, fp8=kind == "fp8", nhd=kind == "nhd")
    acc = np.full((9, 64), 99, np.int32)
    for s, p in enumerate(paths):
        acc[s, :len(p)] = p
    k, v = c.k.clone(), c.v.clone()
    want_k, want_v = k.clone(), v.clone()
    for s, p in enumerate(paths):
        for i, j in enumerate(p):
            a, b = int(L[s] - n[s] + j), int(L[s] - n[s] + i)
            pa, pb = c.tab[s, a // bs], c.tab[s, b // bs]
            want_k[pb, :, b % bs] = k[pa, :, a % bs]
            if kind == "fp8":
                want_v[pb, :, :, b % bs] = v[pa, :, :, a % bs]
            else:
                want_v[pb, :, b % bs] = v[pa, :, a % bs]
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.tree_accept(c.k, c.v, i32(c.tab), i32(L), i32(c.cu), i32(acc), i32([len(p) for p in paths]), workspace=ws)
    assert pdattn.check(ws) == pdattn.OK

    def bits(x):
        return x if kind == "fp8" else x.contiguous().view(torch.int16)
    assert torch.equal(bits(c.k), bits(want_k)) and torch.equal(bits(c.v), bits(want_v))


@pytest.mark.parametrize("fp8", [False, True])
def test_paths_that_are_refused_leave_their_sequence(fp8):
    bs = 16
    n = np.array([8, 8, 8, 8, 8, 8, 8])
    L = np.array([40, 40, 40, 40, 40, 6, 40])
    acc = np.array([[0, 2, 2], [3, 1, 4], [1, 2, 8], [-1, 2, 3], [1, 2, 3], [0, 1, 2], [2, 5, 7]], np.int32)
    count = np.array([3, 3, 3, 3, 9, 2, 3])
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    for s in range(7):
        c = Case(n[s:s + 1], L[s:s + 1], 4, 2, 64, bs, fp8=fp8)
        k = c.k.clone()
        pdattn.tree_accept(c.k, c.v, i32(c.tab), i32(L[s:s + 1]), i32(c.cu), i32(acc[s:s + 1]), i32(count[s:s + 1]), workspace=ws)
        moved = not torch.equal(c.k.view(torch.uint8), k.view(torch.uint8))
        assert pdattn.check(ws) == (pdattn.OK if s == 6 else pdattn.BAD_SEQUENCE) and moved == (s == 6)
    c = Case(n[:1], L[:1], 4, 2, 64, bs, fp8=fp8)
    k, tab = c.k.clone(), c.tab.copy()
    tab[0, 2] = -1
    pdattn.tree_accept(c.k, c.v, i32(tab), i32(L[:1]), i32(c.cu), i32([[5, 6, 7]]), i32([3]), workspace=ws)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX and torch.equal(c.k.view(torch.uint8), k.view(torch.uint8))


# ---------------------------------------------------------------------------------------------------------------
# Trim; rotation positions
# ---------------------------------------------------------------------------------------------------------------
def books(table, lens, NB, bs):
    ref = np.zeros(NB, np.int32)
    for s in range(len(lens)):
        np.add.at(ref, table[s, :-(-max(0, int(lens[s])) // bs)], 1)
    ids = np.flatnonzero(ref == 0)[::-1]
    return ref, np.concatenate([ids, np.full(NB - len(ids), -1)]).astype(np.int32), len(ids)


def test_trim():
    bs, NB, MB = 16, 200, 12
    r = np.random.default_rng(0)
    lens = np.array([100, 64, 65, 0, 1, 192, 30, 48, 17, 33])
    table = np.full((10, MB), -1, np.int32)
    perm = iter(r.permutation(NB))
    for s in range(10):
        table[s, :-(-lens[s] // bs)] = [next(perm) for _ in range(-(-lens[s] // bs))]
    table[7, :2] = table[0, :2]                                # shared pages
    new = np.array([33, 64, 64, 0, 0, 1, 31, 16, -1, 32])      # rows 6 and 8 cannot be served
    ref, free, count = books(table, lens, NB, bs)
    dev = [i32(x) for x in (table, lens, ref, free, [count])]
    ws = pdattn.alloc_pages_workspace(NB, 10)
    pool = pdattn.PagePool(*dev[2:])
    pdattn.pages_trim(pool, dev[0], dev[1], i32(new), bs, ws)
    assert pdattn.check(ws) == pdattn.BAD_SEQUENCE
    for s in range(10):
        if 0 <= new[s] <= lens[s]:
            table[s, -(-new[s] // bs):] = -1
            lens[s] = new[s]
    ref, free, count = books(table, lens, NB, bs)
    for got, want in zip(dev, (table, lens, ref, free, [count])):
        assert (got.cpu().numpy() == want).all()
    pdattn.pages_trim(pool, dev[0], dev[1], dev[1].clone(), bs, ws)          # nothing to do
    assert pdattn.check(ws) == pdattn.OK and (dev[0].cpu().numpy() == table).all() and (dev[3].cpu().numpy() == free).all()
    dev[0][0, 1] = NB + 3                                                   # books and table that do not match
    dev[0][5, 0] = int(free[0])
    pdattn.pages_trim(pool, dev[0], dev[1], torch.zeros_like(dev[1]).where(torch.arange(10, device="cuda") % 5 == 0, dev[1]), bs, ws)
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX


@pytest.mark.parametrize("S", [300, 2500])
def test_trim_of_many_rows(S):
    """Many rows over many pages; every seventh cannot be served."""
    bs, MB = 32, 40
    r = np.random.default_rng(S)
    lens = r.integers(0, MB * bs + 1, S)
    NB = int((-(-lens // bs)).sum()) + 17
    table, perm, at = np.full((S, MB), -1, np.int32), r.permutation(NB), 0
    for s in range(S):
        k = -(-int(lens[s]) // bs)
        table[s, :k], at = perm[at:at + k], at + k
    new = (lens * r.random(S)).astype(np.int64)
    new[::7] = lens[::7] + 1
    ref, free, count = books(table, lens, NB, bs)
    dev = [i32(x) for x in (table, lens, ref, free, [count])]
    ws = pdattn.alloc_pages_workspace(NB, S)
    pdattn.pages_trim(pdattn.PagePool(*dev[2:]), dev[0], dev[1], i32(new), bs, ws)
    assert pdattn.check(ws) == pdattn.BAD_SEQUENCE
    for s in range(S):
        if s % 7:
            lens[s] = new[s]
            table[s, -(-int(new[s]) // bs):] = -1
    ref, free, count = books(table, lens, NB, bs)
    for got, want in zip(dev, (table, lens, ref, free, [count])):
        assert (got.cpu().numpy() == want).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_positions_are_the_callers(fp8, interleaved):
    """A token rotated by position p lands where the cache wants it, with the bits that position p gives elsewhere."""
    S, H, d, bs = 3, 2, 64, 16
    n, L = np.array([5, 1, 4]), np.array([40, 1, 300])
    N = 10
    qkv = torch.randn(N, 4 + 2 * H, d, device="cuda", dtype=BF16)
    q, k, v = qkv[:, :4], qkv[:, 4:4 + H], qkv[:, 4 + H:]
    pos = np.array([35, 36, 36, 37, 100000, 0, 296, 297, 297, -3])
    table = np.arange(S * 19, dtype=np.int32).reshape(S, 19)
    f = (1e6 ** (-torch.arange(0, d, 2, device="cuda") / d)).float()
    scales = (torch.full((H,), 0.05, device="cuda"),) * 2
    dt = torch.uint8 if fp8 else BF16
    kc, vc = torch.zeros(S * 19, H, bs, d, device="cuda", dtype=dt), torch.zeros(S * 19, H, *((d, bs) if fp8 else (bs, d)), device="cuda", dtype=dt)
    out = torch.empty(N, 4, d, device="cuda", dtype=BF16)
    call = pdattn.rope_append_fp8 if fp8 else pdattn.rope_append
    extra = scales if fp8 else ()
    call(q, k, v, out, kc, vc, *extra, i32(table), i32(L), f, cu_tokens=i32([0, 5, 6, 10]), interleaved=interleaved, positions=i32(pos))
    at = [L[s] - n[s] + j for s in range(S) for j in range(n[s])]
    seq = np.repeat(np.arange(S), n)
    for t in range(N):
        if pos[t] < 0:
            continue
        # the same token alone, at a place whose number is its position
        P = int(pos[t]) // bs + 1
        k1 = torch.zeros(1, H, bs, d, device="cuda", dtype=dt)
        v1 = torch.zeros(1, H, *((d, bs) if fp8 else (bs, d)), device="cuda", dtype=dt)
        o1 = torch.empty(1, 4, d, device="cuda", dtype=BF16)
        call(q[t:t + 1], k[t:t + 1], v[t:t + 1], o1, k1, v1, *extra, i32(np.zeros((1, P))), i32([pos[t] + 1]), f, interleaved=interleaved)
        assert torch.equal(out[t], o1[0])
        page, slot = int(table[seq[t], at[t] // bs]), at[t] % bs
        assert torch.equal(kc[page, :, slot], k1[0, :, pos[t] % bs])
        if fp8:
            assert torch.equal(vc[page, :, :, slot], v1[0, :, :, pos[t] % bs])
        else:
            assert torch.equal(vc[page, :, slot], v1[0, :, pos[t] % bs])
    with pytest.raises(ValueError):
        call(q, k, v, out, kc, vc, *extra, i32(table), i32(L), f, cu_tokens=i32([0, 5, 6, 10]), positions=i32(pos[:9]))
