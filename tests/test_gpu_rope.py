"""Rotary positions with the KV append against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def inv_freq(rotary, theta=1e6, factor=1.0):
    f = theta ** (-np.arange(0, rotary, 2) / rotary)
    return torch.from_numpy((f / factor).astype(np.float32)).cuda()


def make(n, L, Hq, Hkv, d, bs, seed=0, fused=True, spare=2, nhd=False):
    """n[s] new tokens of L[s] per sequence; caches filled with a pattern so that every slot that is not written shows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, L = np.asarray(n), np.asarray(L)
    N = int(n.sum())
    pages = np.maximum(0, -(-L // bs))
    MB = int(max(1, pages.max())) + 1
    NB = int(pages.sum()) + spare
    perm = np.random.default_rng(seed).permutation(NB)
    table = np.full((len(n), MB), -1, np.int32)
    at = 0
    for s in range(len(n)):
        table[s, :pages[s]] = perm[at:at + pages[s]]
        at += pages[s]
    if fused:
        qkv = torch.randn(N, Hq + 2 * Hkv, d, device="cuda", dtype=BF16, generator=g)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    else:
        q, k, v = (torch.randn(N, h, d, device="cuda", dtype=BF16, generator=g) for h in (Hq, Hkv, Hkv))
    shape = (NB, bs, Hkv, d) if nhd else (NB, Hkv, bs, d)
    kc, vc = (torch.randn(*shape, device="cuda", dtype=BF16, generator=g) for _ in range(2))
    if nhd:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
    return dict(q=q, k=k, v=v, kc=kc, vc=vc, table=torch.from_numpy(table).cuda(), cu=cu,
                lens=torch.from_numpy(L.astype(np.int32)).cuda(), n=n, L=L, bs=bs, tab=table)


def rotated(x, pos, f, rotary, interleaved, mag):
    """Rows x [m, H, d] at positions pos, in 64 bits, and the size of what was added up (for the bound on fp32 work)."""
    x = x.double().cpu().numpy().copy()
    ang = np.asarray(pos, np.float64)[:, None] * f.double().cpu().numpy()[None]
    c, s = (mag * np.cos(ang))[:, None], (mag * np.sin(ang))[:, None]
    i = np.arange(rotary // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    u, w = x[..., a].copy(), x[..., b].copy()
    size = np.zeros_like(x)
    x[..., a], x[..., b] = u * c - w * s, w * c + u * s
    size[..., a] = size[..., b] = abs(mag) * (abs(u) + abs(w))
    return x, size


def close(got, want, size):
    # one rounding to bf16 (half a step: 2^-8 of the value), and the fp32 work before it: the reduced angle is off by at
    # most 2 pi * 2^-25, sine and cosine by two units, two products and a sum -- below 2^-20 of |x| + |y|
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (abs(got - want) <= 2.0 ** -8 * abs(want) + 2.0 ** -20 * size + 1e-30).all(), abs(got - want).max()


def tokens(c):
    for s in range(len(c["n"])):
        t0 = int(c["n"][:s].sum())
        for j in range(int(c["n"][s])):
            yield s, t0 + j, int(c["L"][s] - c["n"][s] + j)


def check_caches(c, kc0, vc0, want_k, size_k):
    """Written slots hold the rotated k and the very v; every other slot is as before."""
    kc, vc = c["kc"].clone(), c["vc"].clone()
    NB = kc.shape[0]
    got, rows = [], []
    for s, t, pos in tokens(c):
        page = c["tab"][s, pos // c["bs"]] if 0 <= pos and pos // c["bs"] < c["tab"].shape[1] else -1
        if not 0 <= page < NB:
            continue
        slot = pos % c["bs"]
        got.append(kc[page, :, slot].clone())
        rows.append(t)
        assert torch.equal(vc[page, :, slot], c["v"][t])
        kc[page, :, slot] = kc0[page, :, slot]
        vc[page, :, slot] = vc0[page, :, slot]
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)
    if rows:
        close(torch.stack(got), want_k[rows], size_k[rows])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rotary,bs", [(28, 4, 128, 128, 16), (4, 1, 64, 64, 16), (5, 5, 128, 32, 64),
                                               (16, 1, 64, 16, 32), (3, 3, 128, 112, 16), (32, 16, 64, 48, 64)])
def test_ragged(Hq, Hkv, d, rotary, bs, interleaved):
    n = [1, 0, 17, 64, 3, 0, 130]
    L = [1, 9, 17, 100, 70000, 0, 131]
    c = make(n, L, Hq, Hkv, d, bs, seed=Hq)
    f = inv_freq(rotary)
    kc0, vc0 = c["kc"].clone(), c["vc"].clone()
    out = torch.full_like(c["q"].contiguous(), 7.0)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    pdattn.rope_append(c["q"], c["k"], c["v"], out, c["kc"], c["vc"], c["table"], c["lens"], f, cu_tokens=c["cu"],
                       rotary_dim=rotary, interleaved=interleaved, magnitude=1.25, workspace=ws)
    pos = [p for _, _, p in tokens(c)]
    close(out, *rotated(c["q"], pos, f, rotary, interleaved, 1.25))
    check_caches(c, kc0, vc0, *rotated(c["k"], pos, f, rotary, interleaved, 1.25))
    assert int(ws[:4].view(torch.int32)) == 0
    if rotary < d:
        assert torch.equal(out[..., rotary:], c["q"][..., rotary:])


@pytest.mark.parametrize("S,hi", [(1, 5), (256, 9000), (1500, 40)])
def test_one_token_per_sequence(S, hi):
    r = np.random.default_rng(S)
    L = r.integers(1, hi, S)
    c = make(np.ones(S, int), L, 4, 2, 128, 16, seed=S)
    f = inv_freq(128)
    kc0, vc0 = c["kc"].clone(), c["vc"].clone()
    out = torch.empty(S, 4, 128, device="cuda", dtype=BF16)
    pdattn.rope_append(c["q"], c["k"], c["v"], out, c["kc"], c["vc"], c["table"], c["lens"], f)
    close(out, *rotated(c["q"], L - 1, f, 128, False, 1.0))
    check_caches(c, kc0, vc0, *rotated(c["k"], L - 1, f, 128, False, 1.0))
    # the ragged form with one token each is the same call
    c["kc"].copy_(kc0)
    other = torch.empty_like(out)
    pdattn.rope_append(c["q"], c["k"], c["v"], other, c["kc"], c["vc"], c["table"], c["lens"], f, cu_tokens=c["cu"])
    assert torch.equal(out, other)


def test_far_positions_keep_their_angle():
    """Near 2^30 a 32-bit product of position and frequency would be off by tens of radians."""
    L = np.array([2 ** 30 + 7, 2 ** 31 - 9])
    k, v, q = (torch.randn(2, 1, 64, device="cuda", dtype=BF16) for _ in range(3))
    kc, vc = (torch.zeros(1, 1, 16, 64, device="cuda", dtype=BF16) for _ in range(2))
    table = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    out, f = torch.empty_like(q), inv_freq(64)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    pdattn.rope_append(q, k, v, out, kc, vc, table, torch.from_numpy(L.astype(np.int32)).cuda(), f, workspace=ws)
    close(out, *rotated(q, L - 1, f, 64, False, 1.0))
    assert not kc.any() and not vc.any()                      # past the row: not written, and said so
    assert int(ws[:4].view(torch.int32)) == 1


def test_in_place_and_without_queries():
    c = make([3, 5], [20, 5], 4, 2, 128, 16, fused=False)
    f = inv_freq(128)
    out = torch.empty_like(c["q"])
    args = (c["kc"], c["vc"], c["table"], c["lens"], f)
    pdattn.rope_append(c["q"], c["k"], c["v"], out, *args, cu_tokens=c["cu"])
    want = c["kc"].clone()
    c["kc"].zero_()
    pdattn.rope_append(None, c["k"], c["v"], None, *args, cu_tokens=c["cu"])
    written = c["kc"] != 0
    assert torch.equal(c["kc"][written], want[written]) and int(written.sum()) > 8 * 2 * 100
    pdattn.rope_append(c["q"], c["k"], c["v"], c["q"], *args, cu_tokens=c["cu"])
    assert torch.equal(c["q"], out)


def test_bad_pages_short_contexts_and_padding():
    """Sequence 0: a page out of range; 1: more new tokens than its context; 2: past its table row; rows behind the last
    sequence stay as they are."""
    c = make([20, 4, 3], [33, 2, 40], 4, 2, 64, 16)
    c["tab"][0, 1] = c["kc"].shape[0]
    c["tab"][2, 2] = -5
    c["table"] = torch.from_numpy(c["tab"]).cuda()
    pad = 5
    q, k, v = (torch.cat([c[x], torch.randn(pad, c[x].shape[1], 64, device="cuda").to(BF16)]) for x in "qkv")
    out = torch.full_like(q, 7.0)
    kc0, vc0 = c["kc"].clone(), c["vc"].clone()
    f = inv_freq(64)
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.rope_append(q, k, v, out, c["kc"], c["vc"], c["table"], c["lens"], f, cu_tokens=c["cu"], workspace=ws)
    pos = np.array([p for _, _, p in tokens(c)])
    want, size = rotated(c["q"], pos, f, 64, False, 1.0)
    live = np.flatnonzero(pos >= 0)
    close(out[live], want[live], size[live])
    assert not out[np.flatnonzero(pos < 0)].any()
    assert (out[27:] == 7).all()
    check_caches(c, kc0, vc0, *rotated(c["k"], pos, f, 64, False, 1.0))
    assert pdattn.check(ws) == pdattn.BAD_PAGE_INDEX and pdattn.check(ws) == pdattn.OK


def test_token_major_pages():
    c = make([17, 1], [40, 3], 8, 4, 128, 32, nhd=True)
    f = inv_freq(128)
    kc0, vc0 = c["kc"].clone(), c["vc"].clone()
    out = torch.empty_like(c["q"].contiguous())
    pdattn.rope_append(c["q"], c["k"], c["v"], out, c["kc"], c["vc"], c["table"], c["lens"], f, cu_tokens=c["cu"])
    check_caches(c, kc0, vc0, *rotated(c["k"], [p for _, _, p in tokens(c)], f, 128, False, 1.0))


@pytest.mark.parametrize("d,rotary,bs,interleaved", [(128, 128, 16, False), (64, 32, 64, True), (128, 64, 32, False)])
def test_fp8_cache(d, rotary, bs, interleaved):
    n, L, Hq, Hkv = [1, 40, 0, 7], [50, 40, 3, 2000], 6, 3
    c = make(n, L, Hq, Hkv, d, bs)
    NB = c["kc"].shape[0]
    k8, v8 = (torch.randint(0, 120, s, device="cuda", dtype=torch.uint8) for s in ((NB, Hkv, bs, d), (NB, Hkv, d, bs)))
    k0, v0 = k8.clone(), v8.clone()
    ks, vs = torch.tensor([0.004, 0.02, 1.0], device="cuda"), torch.tensor([0.005, 0.1, 3.0], device="cuda")   # the first saturates
    f, out = inv_freq(rotary), torch.empty(48, Hq, d, device="cuda", dtype=BF16)
    pdattn.rope_append_fp8(c["q"], c["k"], c["v"], out, k8, v8, ks, vs, c["table"], c["lens"], f, cu_tokens=c["cu"],
                           rotary_dim=rotary, interleaved=interleaved)
    pos = [p for _, _, p in tokens(c)]
    close(out, *rotated(c["q"], pos, f, rotary, interleaved, 1.0))
    want, size = rotated(c["k"], pos, f, rotary, interleaved, 1.0)
    sc = ks.double().cpu().numpy()[:, None]
    for s, t, p in tokens(c):
        page, slot = c["tab"][s, p // bs], p % bs
        for codes, x, sz, scale in ((k8[page, :, slot], want[t], size[t], sc),
                                    (v8[page, :, :, slot], c["v"][t].double().cpu().numpy(), 0.0, vs.double().cpu().numpy()[:, None])):
            got = codes.contiguous().view(F8).double().cpu().numpy()
            y = x / scale
            # half a step of e4m3 (2^-4 of the value; 2^-10 among the subnormals), decided on the fp32 result
            y = np.clip(y, -448, 448)
            assert (abs(got - y) <= 2.0 ** -4 * abs(y) + 2.0 ** -10 + 2.0 ** -20 * sz / scale).all()
        k8[page, :, slot], v8[page, :, :, slot] = k0[page, :, slot], v0[page, :, :, slot]
    assert torch.equal(k8, k0) and torch.equal(v8, v0)


def test_agrees_with_the_plain_append():
    """Without rotation (zero frequencies) the caches are what pdattn_append_kv writes."""
    c = make([1] * 9, np.arange(1, 10) * 13, 4, 2, 128, 16, fused=False)
    kc, vc, lens = c["kc"].clone(), c["vc"].clone(), c["lens"] - 1
    pdattn.append_kv(c["k"], c["v"], kc, vc, c["table"], lens)
    out = torch.empty_like(c["q"])
    pdattn.rope_append(c["q"], c["k"], c["v"], out, c["kc"], c["vc"], c["table"], c["lens"], torch.zeros(64, device="cuda"))
    assert torch.equal(out, c["q"]) and torch.equal(kc, c["kc"]) and torch.equal(vc, c["vc"]) and torch.equal(lens, c["lens"])


def test_captured_and_replayed():
    c = make([1] * 4, [5, 9, 17, 33], 4, 2, 64, 16)
    f, out = inv_freq(64), torch.zeros(4, 4, 64, device="cuda", dtype=BF16)
    args = (c["q"], c["k"], c["v"], out, c["kc"], c["vc"], c["table"], c["lens"], f)
    pdattn.rope_append(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pdattn.rope_append(*args)
    c["lens"] -= 3                       # the replayed call goes by the lengths of its time
    graph.replay()
    close(out, *rotated(c["q"], np.array([1, 5, 13, 29]), f, 64, False, 1.0))


def test_wrapper_refuses_what_the_library_cannot_see():
    c = make([1] * 4, [5, 9, 17, 33], 4, 2, 64, 16)
    f, out = inv_freq(64), torch.zeros(4, 4, 64, device="cuda", dtype=BF16)
    good = dict(q=c["q"], k_new=c["k"], v_new=c["v"], q_out=out, k_cache=c["kc"], v_cache=c["vc"], block_table=c["table"],
                context_lens=c["lens"], inv_freq=f)
    for name, bad in [("q", c["q"].float()), ("context_lens", c["lens"].long()), ("inv_freq", f.double()), ("v_new", c["v"].cpu())]:
        with pytest.raises((TypeError, ValueError)):
            pdattn.rope_append(**dict(good, **{name: bad}))
    for name, bad in [("block_table", c["table"][:3]), ("inv_freq", f[:7]), ("q_out", out[:2]), ("v_cache", c["vc"][:, :, :, :32]),
                      ("k_new", c["k"].transpose(1, 2).contiguous().transpose(1, 2))]:
        with pytest.raises(ValueError):
            pdattn.rope_append(**dict(good, **{name: bad}))
