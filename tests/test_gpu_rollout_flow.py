"""The operators together, as a rollout uses them: prompts reserved, rotated and appended, attended, forked into groups of
samples, decoded, partly freed, compacted and decoded on.  Every attention output is checked against the definition in 64
bits over the keys and values that were appended, and the caches against those after every page move."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


class Engine:
    def __init__(self, fp8, Hq, Hkv, d, bs, rows, NB, MB, seed):
        self.fp8, self.Hq, self.Hkv, self.d, self.bs = fp8, Hq, Hkv, d, bs
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        dt = torch.uint8 if fp8 else BF16
        self.k = torch.zeros(NB, Hkv, bs, d, device="cuda", dtype=dt)
        self.v = torch.zeros(NB, Hkv, d, bs, device="cuda", dtype=dt) if fp8 else torch.zeros_like(self.k)
        if not fp8:
            self.k.fill_(math.nan)
            self.v.fill_(math.nan)
        self.ks, self.vs = (torch.full((Hkv,), x, device="cuda") for x in (0.03, 0.02))
        self.table = torch.full((rows, MB), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.pool = pdattn.PagePool.create(NB)
        self.pages_ws = pdattn.alloc_pages_workspace(NB, rows)
        self.src, self.dst = (torch.empty(max(NB // 2, rows), dtype=torch.int32, device="cuda") for _ in range(2))
        self.inv_freq = torch.from_numpy((1e4 ** (-np.arange(0, d, 2) / d)).astype(np.float32)).cuda()
        self.scale, self.cap = 1 / math.sqrt(d), 20.0
        self.slopes = (2.0 ** (-torch.arange(Hq, device="cuda") - 3)).float()
        self.kept = {}                       # row -> K and V as they were appended, [Hkv, L, d] in 64 bits

    def i32(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def gathered(self, row):
        L = int(self.lens[row])
        pg = self.table[row, :-(-L // self.bs)].long()
        if self.fp8:
            k = self.k[pg].view(F8).double() * self.ks.double().view(1, -1, 1, 1)
            v = self.v[pg].view(F8).double().transpose(2, 3) * self.vs.double().view(1, -1, 1, 1)
        else:
            k, v = self.k[pg].double(), self.v[pg].double()
        return [x.transpose(0, 1).reshape(self.Hkv, -1, self.d)[:, :L] for x in (k, v)]

    def step(self, new):
        """New tokens for some rows: reserve, rotate and append, attend, check."""
        n = np.array([new.get(r, 0) for r in range(len(self.lens))])
        pdattn.pages_reserve(self.pool, self.table, self.lens, self.i32(n), self.bs, self.pages_ws)
        assert pdattn.check(self.pages_ws) == pdattn.OK
        N, H = int(n.sum()), self.Hq + 2 * self.Hkv
        qkv = torch.randn(N, H, self.d, device="cuda", generator=self.g).to(BF16)
        q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
        qr, out = torch.empty(N, self.Hq, self.d, device="cuda", dtype=BF16), torch.zeros(N, self.Hq, self.d, device="cuda", dtype=BF16)
        cu = self.i32(np.concatenate([[0], np.cumsum(n)]))
        if self.fp8:
            pdattn.rope_append_fp8(q, k, v, qr, self.k, self.v, self.ks, self.vs, self.table, self.lens, self.inv_freq, cu_tokens=cu)
        else:
            pdattn.rope_append(q, k, v, qr, self.k, self.v, self.table, self.lens, self.inv_freq, cu_tokens=cu)
        rows = np.flatnonzero(n)
        if (n[rows] == 1).all():             # single tokens: the active rows as a batch of their own
            at = torch.from_numpy(rows).cuda()
            ws = pdattn.alloc_workspace(len(rows), self.Hq, self.Hkv, self.d, self.bs)
            sc = pdattn.Score(logit_cap=self.cap, bias_slopes=self.slopes)
            args = (self.table[at].contiguous(), self.lens[at].contiguous(), self.scale, out, ws, sc)
            if self.fp8:
                pdattn.decode_scored_fp8(qr, self.k, self.v, self.ks, self.vs, *args)
            else:
                pdattn.decode_scored(qr, self.k, self.v, *args)
            assert pdattn.check(ws) == pdattn.OK
        elif not self.fp8:
            ws = pdattn.alloc_prefill_workspace(len(n), N, self.Hq, self.Hkv, self.d, self.bs)
            pdattn.prefill(qr, self.k, self.v, self.table, self.lens, cu, self.scale, out, ws,
                           score=pdattn.Score(logit_cap=self.cap, bias_slopes=self.slopes))
            assert pdattn.check(ws) == pdattn.OK
        else:
            out = None                       # prompts of an fp8 cache: appended only
        t0, G = 0, self.Hq // self.Hkv
        for r in rows:
            kk, vv = self.gathered(r)
            L, m = kk.shape[1], int(n[r])
            if r in self.kept:               # what was there before is still there
                assert all(torch.equal(a, b[:, :L - m]) for a, b in zip(self.kept[r], (kk, vv)))
            # the appended keys: rotated k, rounded once (to bf16, or to a code of the scale)
            pos = torch.arange(L - m, L, device="cuda").double()
            ang = pos[:, None, None] * self.inv_freq.double()
            a, b = k[t0:t0 + m].double().chunk(2, -1)
            want = torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1).transpose(0, 1)
            step = 2.0 ** -4 if self.fp8 else 2.0 ** -8
            assert ((kk[:, L - m:] - want).abs() <= step * want.abs() + (2.0 ** -10 * 0.03 if self.fp8 else 0) + 2.0 ** -17).all()
            self.kept[r] = (kk, vv)
            if out is not None:
                x = torch.einsum("nhgd,htd->hgnt", qr[t0:t0 + m].double().view(m, self.Hkv, G, self.d), kk) * self.scale
                t = torch.arange(L, device="cuda")
                x = self.cap * torch.tanh(x / self.cap) - self.slopes.double().view(self.Hkv, G, 1, 1) * (pos[:, None] - t).abs()
                p = torch.softmax(torch.where(t <= pos[:, None], x, -math.inf), -1)
                ref = torch.einsum("hgnt,htd->nhgd", p, vv).reshape(m, self.Hq, self.d)
                size = torch.einsum("hgnt,htd->nhgd", p, vv.abs()).reshape(m, self.Hq, self.d)
                # half a bf16 step of the result, bf16 weights at most, fp32 work (2^-12)
                err = (out[t0:t0 + m].double() - ref).abs()
                assert (err <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * size).all()
            t0 += m

    def copy_pages(self, n):
        pdattn.pages_copy(self.k, self.v, self.src[:n], self.dst[:n], workspace=self.pages_ws)
        assert pdattn.check(self.pages_ws) == pdattn.OK
        self.all_kept()

    def all_kept(self):
        for r, (k, v) in self.kept.items():
            assert all(torch.equal(a, b) for a, b in zip((k, v), self.gathered(r)))


@pytest.mark.parametrize("fp8,Hq,Hkv,d,bs", [(False, 8, 2, 128, 16), (False, 4, 4, 64, 32), (True, 8, 2, 128, 16), (True, 6, 2, 64, 64)])
def test_rollout(fp8, Hq, Hkv, d, bs):
    groups, size = 3, 4
    rows = groups * (1 + size)
    e = Engine(fp8, Hq, Hkv, d, bs, rows, NB=200, MB=20, seed=Hq)
    prompts = [5, 130, 3 * bs]               # a partial page, several pages, whole pages only
    e.step({g: prompts[g] for g in range(groups)})
    parents = np.repeat(np.arange(groups), size)
    children = groups + np.arange(groups * size)
    pdattn.pages_fork(e.pool, e.table, e.lens, e.i32(parents), e.i32(children), e.src, e.dst, bs, e.pages_ws)
    for p, c in zip(parents, children):
        e.kept[int(c)] = e.kept[int(p)]
    e.copy_pages(len(parents))
    # the prompts' own rows are done; their whole pages live on in the samples
    pdattn.pages_free(e.pool, e.table, e.lens, e.i32(np.arange(groups)), bs, e.pages_ws)
    for g in range(groups):
        del e.kept[g]
    e.all_kept()
    alive = [int(c) for c in children]
    for _ in range(bs + 2):                  # across a page border for every sample
        e.step({r: 1 for r in alive})
    gone = alive[1::3]
    pdattn.pages_free(e.pool, e.table, e.lens, e.i32(gone), bs, e.pages_ws)
    alive = [r for r in alive if r not in gone]
    for r in gone:
        del e.kept[r]
    pdattn.pages_compact(e.pool, e.table, e.lens, e.src[:100], e.dst[:100], bs, e.pages_ws)
    e.copy_pages(100)
    live = int((e.pool.ref_counts > 0).sum())
    assert bool((e.pool.ref_counts[:live] > 0).all()) and int(e.pool.free_count) == 200 - live
    if not fp8:
        e.step({r: 3 + i for i, r in enumerate(alive)})     # a few tokens at once
    for _ in range(3):
        e.step({r: 1 for r in alive})
    pdattn.pages_free(e.pool, e.table, e.lens, e.i32(alive), bs, e.pages_ws)
    assert pdattn.check(e.pages_ws) == pdattn.OK
    assert int(e.pool.free_count) == 200 and not e.pool.ref_counts.any()


def test_calls_that_overlap_on_streams_of_their_own():
    """Prompt attention of one batch beside the decode steps of another, each with a workspace of its own: the same bits as
    one after the other."""
    g = torch.Generator(device="cuda").manual_seed(3)
    Hq, Hkv, d, bs = 8, 2, 128, 16

    def batch(n, L):
        pages = -(-L // bs)
        NB = int(pages.sum())
        table = np.full((len(n), int(pages.max())), -1, np.int32)
        at = 0
        for s, p in enumerate(pages):
            table[s, :p] = np.arange(at, at + p)
            at += p
        kc, vc = (torch.randn(NB, Hkv, bs, d, device="cuda", generator=g).bfloat16() for _ in range(2))
        q = torch.randn(int(n.sum()), Hq, d, device="cuda", generator=g).bfloat16()
        i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
        return q, kc, vc, i32(table), i32(L), i32(np.concatenate([[0], np.cumsum(n)]))
    a = batch(np.array([900, 40, 300]), np.array([900, 3000, 1200]))
    b = batch(np.ones(60, np.int64), np.arange(1, 61) * 50)
    e = batch(np.array([30]), np.array([9000]))               # cut along the keys
    wa, we = pdattn.alloc_prefill_workspace(3, 1240, Hq, Hkv, d, bs), pdattn.alloc_prefill_workspace(1, 30, Hq, Hkv, d, bs)
    wb = pdattn.alloc_workspace(60, Hq, Hkv, d, bs)
    score = pdattn.Score(logit_cap=20.0, window=700)

    def calls(outs, streams):
        for x, ws, out, st in ((a, wa, outs[0], streams[0]), (e, we, outs[2], streams[2])):
            pdattn.prefill(*x[:6], 0.09, out, ws, score=score, stream=st)
        q, kc, vc, table, lens, _ = b
        pdattn.decode_scored(q, kc, vc, table, lens, 0.09, outs[1], wb, score, stream=streams[1])
    want = [torch.empty_like(x[0]) for x in (a, b, e)]
    calls(want, [None] * 3)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        got = [torch.full_like(x, 7.0) for x in want]
        torch.cuda.synchronize()
        for _ in range(4):
            calls(got, streams)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert pdattn.check(wa) == pdattn.check(wb) == pdattn.check(we) == pdattn.OK
