"""The operators around draft trees and sparse decoding together, as a rollout would use them: pages from the pool, prompts, trees verified
and their paths taken over, then sparse steps; after every step the caches are what a plain decoder's would be."""
import math

import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
HQ, HKV, D, BS = 8, 2, 128, 16


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def rotate(x, pos, f):
    a = torch.as_tensor(pos, device="cuda").double()[:, None] * f.double()
    c, s = a.cos()[:, None], a.sin()[:, None]
    u, w = x.double().chunk(2, -1)
    return torch.cat((u * c - w * s, w * c + u * s), -1)


def attend(q, k, v, hidden, scale):
    G = HQ // HKV
    x = torch.einsum("jhgd,thd->hgjt", q.double().view(-1, HKV, G, D), k.double()) * scale
    p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
    o = torch.einsum("hgjt,thd->jhgd", p, v.double()).reshape(-1, HQ, D)
    return o, torch.einsum("hgjt,thd->jhgd", p, v.double().abs()).reshape(-1, HQ, D)


@pytest.mark.parametrize("fp8", [False, True])
def test_prompts_trees_and_sparse_steps(fp8):
    r = np.random.default_rng(3)
    g = torch.Generator(device="cuda").manual_seed(3)
    S, MB, NB, K = 3, 40, 130, 8
    f = (1e5 ** (-torch.arange(0, D, 2, device="cuda") / D)).float()
    scale = 1 / math.sqrt(D)
    one = torch.full((HKV,), 0.03, device="cuda")
    if fp8:
        kc, vc = torch.zeros(NB, HKV, BS, D, dtype=torch.uint8, device="cuda"), torch.zeros(NB, HKV, D, BS, dtype=torch.uint8, device="cuda")
    else:
        kc, vc = (torch.zeros(NB, HKV, BS, D, dtype=BF16, device="cuda") for _ in range(2))
    caches = (kc, vc, one, one) if fp8 else (kc, vc)
    pool = pdattn.PagePool.create(NB)
    table = torch.full((S, MB), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    pages_ws = pdattn.alloc_pages_workspace(NB, S)
    tree_ws = pdattn.alloc_tree_workspace(HQ, HKV, D, BS)
    ws, sel_ws = pdattn.alloc_workspace(S, HQ, HKV, D, BS), pdattn.alloc_select_workspace(S, HKV, MB)
    summary = pdattn.PageSummary.create(NB, HKV, D)
    keys, values = ([torch.zeros(0, HKV, D, device="cuda", dtype=torch.double) for _ in range(S)] for _ in range(2))

    def stored(x):                                             # what the cache holds of rows x: rounded once
        return ((x / one[0].double()).clamp(-448, 448).float().to(F8).double() * one[0].double()) if fp8 else x.to(BF16).double()

    def append(q, k, v, cu, positions=None):
        out = torch.empty(q.shape, dtype=BF16, device="cuda")
        call = pdattn.rope_append_fp8 if fp8 else pdattn.rope_append
        call(q, k, v, out, *caches, table, lens, f, cu_tokens=cu, positions=positions)
        return out

    def news(n):
        return [torch.randn(n, h, D, device="cuda", dtype=BF16, generator=g) for h in (HQ, HKV, HKV)]

    def close(got, want, size, why):
        # the result 2^-8 of it; bf16 weights 2^-8 of each; rows rotated by the library (fp32) and here (fp64) may be rounded the other
        # way, a step of bf16 or e4m3 in single elements: below 2^-6 of sum p |v| in all
        err = (got.double() - want).abs()
        assert (err <= 2.0 ** -8 * want.abs() + 2.0 ** -6 * size + 1e-6).all(), (why, float((err / (size + 1e-6)).max()))

    # prompts
    n = np.array([200, 37, 90])
    pdattn.pages_reserve(pool, table, lens, i32(n), BS, pages_ws)
    cu = i32(np.concatenate([[0], np.cumsum(n)]))
    q, k, v = news(int(n.sum()))
    append(q, k, v, cu)
    pdattn.summarize_append(kc, summary, table, lens, cu_tokens=cu, num_tokens=int(n.sum()), k_scale=one if fp8 else None)
    at = 0
    for s in range(S):
        keys[s] = rotate(k[at:at + n[s]], np.arange(n[s]), f)
        values[s] = v[at:at + n[s]].double()
        at += n[s]
    # rounds of drafts: reserve, append at the tokens' depths, attend, take a path over, give the rest back
    for _ in range(4):
        n = r.integers(1, 13, S)
        parents = [[int(r.integers(-1, j)) if j else -1 for j in range(x)] for x in n]
        depth, masks = [], []
        for p in parents:
            dd, mm = [], []
            for j, x in enumerate(p):
                dd.append(0 if x < 0 else dd[x] + 1)
                mm.append((mm[x] if x >= 0 else 0) | 1 << j)
            depth.append(dd)
            masks.append(mm)
        pdattn.pages_reserve(pool, table, lens, i32(n), BS, pages_ws)
        cu = i32(np.concatenate([[0], np.cumsum(n)]))
        q, k, v = news(int(n.sum()))
        pos = np.concatenate([len(keys[s]) + np.array(depth[s]) for s in range(S)])
        qr = append(q, k, v, cu, i32(pos))
        out = torch.empty_like(qr)
        rest = (table, lens, cu, torch.tensor(sum(masks, []), device="cuda"), scale, out, tree_ws)
        (pdattn.decode_tree_fp8 if fp8 else pdattn.decode_tree)(qr, *caches, *rest, max_tree_tokens=int(n.max()))
        kr = rotate(k, pos, f)
        paths, at = [], 0
        for s in range(S):
            kk = stored(torch.cat((keys[s], kr[at:at + n[s]])))
            vv = stored(torch.cat((values[s], v[at:at + n[s]].double())))
            h = len(keys[s])
            hidden = torch.ones(n[s], h + n[s], dtype=torch.bool, device="cuda")
            hidden[:, :h] = False
            for j in range(n[s]):
                for i in range(n[s]):
                    hidden[j, h + i] = not masks[s][j] >> i & 1
            close(out[at:at + n[s]], *attend(rotate(q[at:at + n[s]], pos[at:at + n[s]], f).to(BF16), kk, vv, hidden, scale), "tree")
            j, path = int(r.integers(0, n[s])), []
            while j >= 0:
                path.insert(0, j)
                j = parents[s][j]
            paths.append(path)
            keys[s], values[s] = (torch.cat((x, y[at:at + n[s]][path].double())) for x, y in ((keys[s], kr), (values[s], v)))
            at += n[s]
        acc = np.full((S, 13), -1, np.int32)
        for s, p in enumerate(paths):
            acc[s, :len(p)] = p
        pdattn.tree_accept(kc, vc, table, lens, cu, i32(acc), i32([len(p) for p in paths]), workspace=ws)
        new = i32([len(x) for x in keys])
        pdattn.pages_trim(pool, table, lens, new, BS, pages_ws)
        # summaries of the pages that the accepted tokens filled
        pdattn.summarize_append(kc, summary, table, lens, cu_tokens=i32(np.concatenate([[0], np.cumsum([len(p) for p in paths])])),
                                num_tokens=sum(map(len, paths)), k_scale=one if fp8 else None, workspace=ws)
        assert (lens.cpu().numpy() == [len(x) for x in keys]).all()
        assert int(pool.free_count) == NB - sum(-(-len(x) // BS) for x in keys)
    # sparse steps
    for _ in range(20):
        pdattn.pages_reserve(pool, table, lens, i32(np.ones(S)), BS, pages_ws)
        q, k, v = news(S)
        pos = np.array([len(x) for x in keys])
        qr = append(q, k, v, None)
        kr = rotate(k, pos, f)
        pdattn.summarize_append(kc, summary, table, lens, k_scale=one if fp8 else None, workspace=ws)
        sel = torch.empty(S, HKV, K, dtype=torch.int32, device="cuda")
        pdattn.select_pages(qr, summary, table, lens, sel, BS, sel_ws, num_first=1, num_recent=2)
        out = torch.empty_like(qr)
        (pdattn.decode_selected_fp8 if fp8 else pdattn.decode_selected)(qr, *caches, table, lens, sel, scale, out, ws)
        chosen = sel.cpu().numpy()
        for s in range(S):
            keys[s], values[s] = torch.cat((keys[s], kr[s:s + 1])), torch.cat((values[s], v[s:s + 1].double()))
            L = len(keys[s])
            for h in range(HKV):
                b = chosen[s, h][chosen[s, h] >= 0]
                P = -(-L // BS)
                assert len(set(b)) == len(b) == min(P, K) and (np.diff(b) > 0).all() and b[0] == 0 and b[-1] == P - 1
                hidden = torch.ones(1, L, dtype=torch.bool, device="cuda")
                for x in b:
                    hidden[:, x * BS:x * BS + BS] = False
                o, size = attend(rotate(q[s:s + 1], pos[s:s + 1], f).to(BF16), stored(keys[s]), stored(values[s]), hidden, scale)
                sl = slice(h * HQ // HKV, (h + 1) * HQ // HKV)
                close(out[s:s + 1, sl], o[:, sl], size[:, sl], "sparse")
    for w in (pages_ws, tree_ws, ws, sel_ws):
        assert pdattn.check(w) == pdattn.OK
