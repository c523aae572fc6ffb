"""Page bookkeeping: every operation against a plain model of the books, entry for entry."""
import numpy as np
import pytest
import torch

from paper_2607_09207_b200 import pdattn

pytestmark = pytest.mark.gpu


class Books:
    """The plain model: lists and loops."""

    def __init__(self, NB, S, MB, bs):
        self.NB, self.S, self.MB, self.bs = NB, S, MB, bs
        self.table = np.full((S, MB), -1, np.int32)
        self.lens = np.zeros(S, np.int32)
        self.ref = np.zeros(NB, np.int32)

    def free_list(self):
        ids = np.flatnonzero(self.ref == 0)[::-1]
        return np.concatenate([ids, np.full(self.NB - len(ids), -1)]).astype(np.int32), len(ids)

    def pages(self, s):
        return -(-int(self.lens[s]) // self.bs)

    def take(self, k):
        ids = np.flatnonzero(self.ref == 0)[:k]
        self.ref[ids] = 1
        return ids

    def reserve(self, new):
        ok = [n >= 0 and self.lens[s] + n <= self.MB * self.bs for s, n in enumerate(new)]
        need = [-(-(int(self.lens[s]) + int(n)) // self.bs) - self.pages(s) if ok[s] else 0 for s, n in enumerate(new)]
        if sum(need) > (self.ref == 0).sum():
            return pdattn.OUT_OF_PAGES
        for s, n in enumerate(new):
            if ok[s]:
                at = self.pages(s)
                self.table[s, at:at + need[s]] = self.take(need[s])
                self.lens[s] += n
        return pdattn.OK if all(ok) else pdattn.BAD_SEQUENCE

    def fork(self, parents, children):
        n = len(parents)
        none = (np.full(n, -1, np.int32),) * 2
        if (any(not (0 <= p < self.S and 0 <= c < self.S) for p, c in zip(parents, children)) or len(set(children)) < n
                or any(self.lens[c] for c in children)):
            return pdattn.BAD_SEQUENCE, none
        L = [int(self.lens[p]) for p in parents]
        if sum(x % self.bs != 0 for x in L) > (self.ref == 0).sum():
            return pdattn.OUT_OF_PAGES, none
        pairs = []
        for p, c, x in zip(parents, children, L):
            whole = x // self.bs
            row = np.full(self.MB, -1, np.int32)
            row[:whole] = self.table[p, :whole]
            np.add.at(self.ref, row[:whole], 1)
            if x % self.bs:
                row[whole] = self.take(1)[0]
                pairs.append((self.table[p, whole], row[whole]))
            self.table[c], self.lens[c] = row, x
        return pdattn.OK, tuple(np.array([x[i] for x in pairs] + [-1] * (n - len(pairs)), np.int32) for i in (0, 1))

    def free(self, seqs):
        bad = False
        for s in seqs:
            if not 0 <= s < self.S:
                bad = True
                continue
            np.subtract.at(self.ref, self.table[s, :self.pages(s)], 1)
            if self.lens[s]:
                self.table[s] = -1
            self.lens[s] = 0
        return pdattn.BAD_SEQUENCE if bad else pdattn.OK

    def compact(self):
        live = np.flatnonzero(self.ref > 0)
        n = len(live)
        src, dst = live[live >= n], np.setdiff1d(np.arange(n), live)
        to = np.arange(self.NB)
        to[src] = dst
        for s in range(self.S):
            self.table[s, :self.pages(s)] = to[self.table[s, :self.pages(s)]]
        self.ref[dst] = self.ref[src]
        self.ref[src] = 0
        fill = np.full(self.NB // 2 - len(src), -1)
        return [np.concatenate([x, fill]).astype(np.int32) for x in (src, dst)]


class Device:
    def __init__(self, m):
        self.m = m
        self.pool = pdattn.PagePool.create(m.NB)
        self.table = torch.from_numpy(m.table.copy()).cuda()
        self.lens = torch.from_numpy(m.lens.copy()).cuda()
        self.ws = pdattn.alloc_pages_workspace(m.NB, m.S)
        self.src, self.dst = (torch.zeros(max(m.NB // 2, m.S), dtype=torch.int32, device="cuda") for _ in range(2))

    def i32(self, x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

    def reserve(self, new):
        pdattn.pages_reserve(self.pool, self.table, self.lens, self.i32(new), self.m.bs, self.ws)
        return pdattn.check(self.ws)

    def fork(self, p, c):
        pdattn.pages_fork(self.pool, self.table, self.lens, self.i32(p), self.i32(c), self.src, self.dst, self.m.bs, self.ws)
        return pdattn.check(self.ws), tuple(x[:len(p)].cpu().numpy() for x in (self.src, self.dst))

    def free(self, s):
        pdattn.pages_free(self.pool, self.table, self.lens, self.i32(s), self.m.bs, self.ws)
        return pdattn.check(self.ws)

    def compact(self):
        k = self.m.NB // 2
        pdattn.pages_compact(self.pool, self.table, self.lens, self.src[:k], self.dst[:k], self.m.bs, self.ws)
        assert pdattn.check(self.ws) == pdattn.OK
        return [x[:k].cpu().numpy() for x in (self.src, self.dst)]

    def same(self):
        m = self.m
        assert np.array_equal(self.table.cpu().numpy(), m.table)
        assert np.array_equal(self.lens.cpu().numpy(), m.lens)
        assert np.array_equal(self.pool.ref_counts.cpu().numpy(), m.ref)
        free, n = m.free_list()
        assert int(self.pool.free_count) == n
        assert np.array_equal(self.pool.free_list.cpu().numpy(), free)


def equal_pairs(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


def test_reserve_fork_free_compact_by_hand():
    m = Books(12, 6, 4, 16)
    d = Device(m)
    d.same()
    assert d.reserve([20, 16, 0, 0, 0, 0]) == m.reserve([20, 16, 0, 0, 0, 0]) == pdattn.OK
    d.same()
    assert m.table[0, :2].tolist() == [0, 1] and m.table[1, 0] == 2
    for p, c in (([0, 1, 0], [3, 4, 5]),):
        a, b = d.fork(p, c), m.fork(p, c)
        assert a[0] == b[0] == pdattn.OK and equal_pairs(a[1], b[1])
        assert b[1][0].tolist() == [1, 1, -1] and b[1][1].tolist() == [3, 4, -1]
    d.same()
    assert d.free([0, 1]) == m.free([0, 1]) == pdattn.OK
    d.same()
    assert equal_pairs(d.compact(), m.compact())
    d.same()
    assert d.free([3, 4, 5, 5, 3]) == m.free([3, 4, 5, 5, 3]) == pdattn.OK     # a row named twice is freed once
    d.same()
    assert m.ref.sum() == 0


def test_refusals_change_nothing():
    m = Books(7, 5, 3, 16)
    d = Device(m)
    assert d.reserve([17, 5, 48, 0, 0]) == m.reserve([17, 5, 48, 0, 0]) == pdattn.OK      # 2 + 1 + 3 of 7 pages
    d.same()
    assert d.reserve([32, 5, 0, 1, -1]) == m.reserve([32, 5, 0, 1, -1]) == pdattn.BAD_SEQUENCE   # rows 0 and 4 refused
    d.same()
    assert m.lens.tolist() == [17, 10, 48, 1, 0]
    assert d.reserve([16, 0, 0, 0, 0]) == m.reserve([16, 0, 0, 0, 0]) == pdattn.OUT_OF_PAGES
    d.same()
    for p, c, why in [([0, 1], [4, 4], pdattn.BAD_SEQUENCE), ([0], [1], pdattn.BAD_SEQUENCE), ([5], [4], pdattn.BAD_SEQUENCE),
                      ([0], [-1], pdattn.BAD_SEQUENCE), ([0], [4], pdattn.OUT_OF_PAGES)]:
        a, b = d.fork(p, c), m.fork(p, c)
        assert a[0] == b[0] == why and equal_pairs(a[1], b[1])
        d.same()
    a, b = d.fork([2], [4]), m.fork([2], [4])          # whole pages only: no page of its own is needed
    assert a[0] == b[0] == pdattn.OK and equal_pairs(a[1], b[1])
    d.same()
    assert d.free([0, 9, -1]) == m.free([0, 9, -1]) == pdattn.BAD_SEQUENCE
    d.same()


def test_books_that_do_not_match_the_table():
    """A row that names a page without references, or none at all, frees nothing and is reported."""
    m = Books(9, 2, 3, 16)
    d = Device(m)
    assert d.reserve([33, 10]) == m.reserve([33, 10])
    d.table[0, 1], d.table[0, 2] = 8, 100
    assert d.free([0]) == pdattn.BAD_PAGE_INDEX
    assert d.pool.ref_counts.cpu().tolist() == [0, 1, 1, 1, 0, 0, 0, 0, 0]
    assert int(d.pool.free_count) == 6 and d.lens.tolist() == [0, 10]
    d.table[1, 0] = 8                                   # not a live page: compaction leaves the entry, and says so
    pdattn.pages_compact(d.pool, d.table, d.lens, d.src[:4], d.dst[:4], 16, d.ws)
    assert pdattn.check(d.ws) == pdattn.BAD_PAGE_INDEX and int(d.table[1, 0]) == 8


@pytest.mark.parametrize("NB,S,MB,bs,seed", [(40, 9, 6, 16, 0), (500, 70, 20, 32, 1), (1, 2, 1, 64, 2), (5003, 1300, 9, 16, 3),
                                            (40001, 300, 300, 64, 4)])
def test_random_sequences_of_operations(NB, S, MB, bs, seed):
    r = np.random.default_rng(seed)
    m = Books(NB, S, MB, bs)
    d = Device(m)
    for step in range(25):
        what = r.integers(0, 5)
        if what <= 1:
            new = r.integers(0, max(2, min(MB * bs, 2 * NB * bs // S)) // (1 if step < 2 else 4) + 1, S) * (r.random(S) < 0.5)
            assert d.reserve(new) == m.reserve(new)
        elif what == 2:
            empty = np.flatnonzero(m.lens == 0)
            n = int(r.integers(0, len(empty) + 1))
            if n:
                c = r.permutation(empty)[:n]
                p = r.integers(0, S, n)
                a, b = d.fork(p, c), m.fork(p, c)
                assert a[0] == b[0] and equal_pairs(a[1], b[1])
        elif what == 3:
            s = r.integers(0, S, int(r.integers(0, S)) // 2 + 1)
            assert d.free(s) == m.free(s) == pdattn.OK
        else:
            assert equal_pairs(d.compact(), m.compact())
        d.same()


@pytest.mark.parametrize("layout", ["head", "token", "head_outermost", "fp8"])
def test_copy(layout):
    NB, H, bs, dim = 300, 3, 32, 64
    if layout == "fp8":
        k, v = (torch.randint(0, 256, s, dtype=torch.uint8, device="cuda") for s in ((NB, H, bs, dim), (NB, H, dim, bs)))
    else:
        shape, order = {"head": ((NB, H, bs, dim), (0, 1, 2, 3)), "token": ((NB, bs, H, dim), (0, 2, 1, 3)),
                        "head_outermost": ((H, NB, bs, dim), (1, 0, 2, 3))}[layout]
        k, v = (torch.randn(*shape, device="cuda").bfloat16().permute(order) for _ in range(2))
    perm = torch.randperm(NB, dtype=torch.int32, device="cuda")
    src, dst = perm[:100].clone(), perm[100:200].clone()
    src[:30] = src[30]                                  # one page to many
    src[40], dst[50] = -1, -1                           # pairs that are skipped
    src[60] = dst[60]                                   # a page onto itself
    k0, v0 = k.clone(), v.clone()
    live = (src >= 0) & (dst >= 0)
    k0[dst[live].long()], v0[dst[live].long()] = k0[src[live].long()], v0[src[live].long()]
    ws = torch.zeros(8448, dtype=torch.uint8, device="cuda")
    pdattn.pages_copy(k, v, src, dst, workspace=ws)
    assert torch.equal(k, k0) and torch.equal(v, v0) and pdattn.check(ws) == pdattn.OK
    src[3], dst[4] = NB, NB + 7                         # out of range: not copied, and said so
    src[0], dst[0] = src[1], src[1]
    src[1:3], src[5:] = -1, -1
    pdattn.pages_copy(k, v, src, dst, workspace=ws)
    assert torch.equal(k, k0) and torch.equal(v, v0) and pdattn.check(ws) == pdattn.BAD_PAGE_INDEX


def test_copy_far_into_a_large_pool():
    """Offsets past 2^32 bytes: the last page of a pool of 5 GB."""
    NB, H, bs, dim = 20000, 8, 64, 128                  # 128 KB a page and cache: 2.6 GB each
    k = torch.zeros(NB, H, bs, dim, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros(2 * NB, H, bs, dim, device="cuda", dtype=torch.bfloat16)[:NB]
    k[0], v[0] = 1.0, 2.0
    big = torch.zeros(2 * NB, H, bs, dim, device="cuda", dtype=torch.bfloat16)
    i = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    pdattn.pages_copy(k, v, i(0), i(NB - 1))
    assert bool((k[NB - 1] == 1).all()) and bool((v[NB - 1] == 2).all()) and not k[1:NB - 1].any()
    big[0] = 3.0
    pdattn.pages_copy(big, big, i(0), i(2 * NB - 1))
    assert bool((big[-1] == 3).all()) and not big[1:-1].any()


def test_captured_and_replayed():
    """A whole cycle in a graph: the same books after every replay from the same state."""
    m = Books(64, 8, 6, 16)
    d = Device(m)
    new, p, c, gone = d.i32([33, 20, 0, 0, 0, 0, 0, 0]), d.i32([0, 1, 0]), d.i32([2, 3, 4]), d.i32([0, 2])

    def cycle():
        pdattn.pages_reserve(d.pool, d.table, d.lens, new, 16, d.ws)
        pdattn.pages_fork(d.pool, d.table, d.lens, p, c, d.src, d.dst, 16, d.ws)
        pdattn.pages_free(d.pool, d.table, d.lens, gone, 16, d.ws)
        pdattn.pages_compact(d.pool, d.table, d.lens, d.src, d.dst, 16, d.ws)
        pdattn.pages_free(d.pool, d.table, d.lens, d.i_all, 16, d.ws)
    d.i_all = d.i32(np.arange(8))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cycle()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cycle()
    for _ in range(3):
        graph.replay()
    assert pdattn.check(d.ws) == pdattn.OK
    d.same()                                            # everything was freed: the books of an empty pool


@pytest.mark.parametrize("dead", [1, 2])
def test_a_dead_page_below_the_live_ones_is_reported_by_compaction(dead):
    """Rows 0 and 1 hold pages 0 and 3, pages 1 and 2 are free; an entry that names one of those is left and reported."""
    m = Books(9, 4, 3, 16)
    d = Device(m)
    assert d.reserve([16, 32, 16, 16]) == m.reserve([16, 32, 16, 16])       # pages 0; 1, 2; 3; 4
    assert d.free([1]) == m.free([1])
    d.table[3, 0] = dead                                # page 4 of row 3 is now nobody's; pages 0, 3, 4 are live
    pdattn.pages_compact(d.pool, d.table, d.lens, d.src[:4], d.dst[:4], 16, d.ws)
    assert pdattn.check(d.ws) == pdattn.BAD_PAGE_INDEX
    assert d.table[:, 0].tolist() == [0, -1, 1, dead]   # page 3 moved to 1, page 4 to 2
    assert pdattn.check(d.ws) == pdattn.OK


def test_requests_whose_total_passes_32_bits_are_refused():
    """1024 rows of 2^21 pages each: 2^31 pages in all."""
    NB, S, MB, bs = 64, 1025, 1 << 21, 16
    pool = pdattn.PagePool.create(NB)
    table = torch.full((S, MB), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    ws = pdattn.alloc_pages_workspace(NB, S)
    for rows, new in ((1024, MB * bs), (1025, MB * bs), (1024, MB * bs - 15)):
        ask = torch.zeros_like(lens)
        ask[:rows] = new
        pdattn.pages_reserve(pool, table, lens, ask, bs, ws)
        assert pdattn.check(ws) == pdattn.OUT_OF_PAGES
        assert int(pool.free_count) == NB and not lens.any() and not pool.ref_counts.any()
        assert pool.free_list.tolist() == list(range(NB - 1, -1, -1))
    assert bool((table[::100] == -1).all())


def test_lengths_stay_within_32_bits():
    """A row wide enough for 2^31 tokens: the request that would pass the largest length is refused, the one before it served."""
    MB, bs, top = 1 << 27, 16, 2 ** 31 - 1
    pool, ws = pdattn.PagePool.create(8), pdattn.alloc_pages_workspace(8, 1)
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((1, MB), -1, dtype=torch.int32, device="cuda")
    lens = i32(top - 40)
    pdattn.pages_reserve(pool, table, lens, i32(41), bs, ws)
    assert pdattn.check(ws) == pdattn.BAD_SEQUENCE and int(lens) == top - 40 and int(pool.free_count) == 8
    pdattn.pages_reserve(pool, table, lens, i32(40), bs, ws)
    assert pdattn.check(ws) == pdattn.OK and int(lens) == top and int(pool.free_count) == 6
    assert table[0, -4:].tolist() == [-1, -1, 0, 1]
