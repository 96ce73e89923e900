"""GPU checks of the calls on pages against the oracle's, which take one list entry
after the other: tables, lengths, counts and page contents are equal.  And a run of
all of them together with cp_kv_append and cp_attn_paged, as a serving loop would."""

import numpy as np
import pytest
import torch

from oracle.pages import Pool
from paper_2609_04774_amd import cpattn as cp

from paged_cases import B, D, DEV, compare, f64, randn
from oracle import window as owin

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Both:
    """A pool on the GPU and the oracle's."""

    def __init__(self, n_seqs, width, n_pages, n_caches=2, Hkv=2, seed=0, dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        self.tables = torch.full((n_seqs, width), -1, dtype=torch.int32, device=DEV)
        self.kv_len, self.refs = i32([0] * n_seqs), i32([0] * n_pages)
        self.caches = [torch.randint(-99, 99, (n_pages, B, Hkv, D), generator=g).to(dtype).to(DEV) for _ in range(n_caches)]
        self.pool = cp.KVPool(self.tables, self.kv_len, self.refs, self.caches)
        self.missing = i32([-7])
        self.want = Pool(self.tables.tolist(), [0] * n_seqs, [0] * n_pages, [c.float().cpu().numpy() for c in self.caches])

    def check(self, missing=None):
        torch.cuda.synchronize()
        assert self.tables.tolist() == self.want.tables
        assert self.kv_len.tolist() == self.want.kv_len
        assert self.refs.tolist() == self.want.refs
        assert self.want.consistent()
        for c, w in zip(self.caches, self.want.caches):
            assert np.array_equal(c.float().cpu().numpy(), w)
        if missing is not None:
            assert self.missing.tolist() == [missing]

    def reserve(self, seqs, add):
        cp.kv_reserve(self.pool, i32(seqs), i32(add), self.missing)
        self.check(self.want.reserve(seqs, add))

    def fork(self, parents, children):
        cp.kv_fork(self.pool, i32(parents), i32(children), self.missing)
        self.check(self.want.fork(parents, children))

    def free(self, seqs, begin, end):
        cp.kv_free(self.pool, i32(seqs), i32(begin), i32(end))
        self.want.free(seqs, begin, end)
        self.check()

    def compact(self):
        ws = torch.empty(cp.kv_compact_workspace_size(self.pool), dtype=torch.uint8, device=DEV)
        cp.kv_compact(self.pool, ws)
        self.want.compact()
        self.check()


def test_reserve():
    b = Both(6, 8, 40)
    b.reserve([3, 0, 5], [17, 16, 1])
    b.reserve([0, 3, 5, 1], [0, 14, 15, 128])         # within a page, to its end, a whole table
    b.reserve([2, 2, -1, 6, 4], [5, 100, 3, 3, 0])    # named again, and outside
    b.reserve([1, 4], [1, -5])                        # a full table, a negative length


def test_reserve_until_the_pages_run_out():
    b = Both(5, 16, 10)
    b.reserve([0, 1, 2, 3, 4], [64, 64, 48, 16, 0])   # 4 + 4 of 10, then 3, 1 and 0
    b.free([0], [0], [64])
    b.reserve([2, 3], [48, 16])


def test_fork_and_free():
    b = Both(12, 8, 60, n_caches=4, seed=1)
    b.reserve([0, 1, 2], [37, 48, 5])
    b.fork([0, 0, 1, 2, 3], [4, 5, 6, 7, 8])          # parts of pages, whole pages, an empty parent
    b.fork([4, 6, 99, 0, 1], [9, 9, 10, -1, 12])      # named again, and outside
    b.fork([0, 10], [10, 11])                         # a child that is a parent
    b.free([0, 5], [0, 16], [37, 40])                 # shared pages stay
    b.free([4, 4, 12, -1, 9], [0, 0, 0, 0, 36], [37, 10, 5, 5, 37])
    b.free([6, 1, 2], [0, 3, 0], [47, 48, 4])         # not the last page; from a page's middle; nothing
    b.free([6], [0], [2**31 - 1])


def test_fork_of_a_parent_whose_pages_are_partly_gone():
    b = Both(6, 8, 40, seed=9)
    b.reserve([0, 1], [70, 45])
    b.free([0, 1], [16, 32], [64, 45])                # pages in the middle; the last one, filled in part
    b.fork([0, 1], [2, 3])


def test_fork_without_pages_left():
    b = Both(6, 4, 5, seed=2)
    b.reserve([0, 1], [20, 32])                       # 4 of 5 pages
    b.fork([0, 0, 1], [2, 3, 4])                      # one copy is left; the last needs none


def test_lists_of_every_length():
    rng = np.random.RandomState(3)
    for n in (1, 2, 63, 300, 1025, 4096):
        b = Both(n + 8, 4, 2 * n + 30, n_caches=1, Hkv=1, seed=n)
        seqs = rng.permutation(n + 8)[:n].tolist()
        b.reserve(seqs, rng.randint(0, 34, n).tolist())
        b.free(seqs[::-1], rng.randint(-5, 20, n).tolist(), rng.randint(0, 40, n).tolist())
    empty = i32([])
    cp.kv_reserve(b.pool, empty, empty, b.missing)
    b.check(0)
    cp.kv_fork(b.pool, empty, empty, b.missing)
    cp.kv_free(b.pool, empty, empty, empty)
    b.check(0)


def test_a_large_pool():
    """Free pages far behind the front, and moves over the whole pool."""
    n = 50000
    b = Both(40, 1300, n, n_caches=1, Hkv=1, seed=4)
    b.reserve(list(range(38)), [20800 - 16 * s for s in range(38)])   # nearly all of it
    b.reserve([38, 39], [500, 77])
    b.free(list(range(0, 36)), [320] * 36, [19000] * 36)
    b.compact()
    b.reserve([39, 2], [100, 3])


@pytest.mark.parametrize("seed", range(4))
def test_random_histories(seed):
    rng = np.random.RandomState(20 + seed)
    n_seqs, n_pages = 20, 120
    b = Both(n_seqs, 12, n_pages, n_caches=3, Hkv=1, seed=seed)
    for _ in range(25):
        what = rng.randint(4)
        n = rng.randint(1, 8)
        seqs = rng.randint(-1, n_seqs + 1, n).tolist()
        if what == 0:
            b.reserve(seqs, rng.randint(-1, 60, n).tolist())
        elif what == 1:
            empty = [s for s in range(n_seqs) if all(p == -1 for p in b.want.tables[s])]
            children = rng.permutation(empty)[:n].tolist()
            b.fork(rng.randint(0, n_seqs, len(children)).tolist(), children)
        elif what == 2:
            begin = rng.randint(-10, 60, n)
            b.free(seqs, begin.tolist(), (begin + rng.randint(0, 150, n)).tolist())
        else:
            b.compact()


def test_compact_borders():
    b = Both(2, 8, 9, seed=5)
    b.compact()                        # nothing in use
    b.reserve([0, 1], [100, 32])       # all but none free
    b.compact()
    b.free([0], [0], [64])
    b.compact()
    cp.kv_compact(cp.KVPool(b.tables, b.kv_len, b.refs), torch.empty(4096, dtype=torch.uint8, device=DEV))  # no caches
    b.check()


@pytest.mark.parametrize("n", [1, 7, 300])
def test_copy_pages(n):
    g = torch.Generator().manual_seed(n)
    for n_caches, shape, dtype in ((1, (16, 1, 8), torch.bfloat16), (6, (16, 8, 128), torch.bfloat16), (2, (48,), torch.int8)):
        caches = [torch.randint(-99, 99, (2 * n + 4, *shape), generator=g).to(dtype).to(DEV) for _ in range(n_caches)]
        perm = torch.randperm(2 * n + 4, generator=g).to(torch.int32)
        src, dst = perm[:n].clone(), perm[n:2 * n].clone()
        want = [c.clone() for c in caches]
        for c in want:
            c[dst.long().to(DEV)] = c[src.long().to(DEV)]
        bad = torch.tensor([-1, 3, 2 * n + 4, 2**31 - 1], dtype=torch.int32)
        cp.kv_copy_pages(caches, torch.cat([src, bad]).to(DEV), torch.cat([dst, bad.flip(0)]).to(DEV))
        # (3 -> 2 n + 4 and 2 n + 4 -> 3 name a page outside)
        assert all(torch.equal(a, b) for a, b in zip(caches, want))


def test_captured_pages():
    """Reserve, append and free in a captured step, replayed."""
    b = Both(4, 20, 64, seed=6)
    b.reserve([0, 1, 2, 3], [30, 16, 1, 47])
    seqs, one, begin = i32([0, 1, 2, 3]), i32([1, 1, 1, 1]), i32([16] * 4)
    end = i32([0] * 4)
    rows = torch.ones(4, 2, D, dtype=torch.bfloat16, device=DEV)
    kv = cp.PagedKV(b.caches[0], b.caches[1], b.tables, b.kv_len)
    ws = torch.empty(cp.kv_compact_workspace_size(b.pool), dtype=torch.uint8, device=DEV)

    def step():
        cp.kv_reserve(b.pool, seqs, one, b.missing)
        cp.kv_append(kv, rows, rows)
        torch.sub(b.kv_len, 24, out=end)
        cp.kv_free(b.pool, seqs, begin, end)
        cp.kv_compact(b.pool, ws)

    def expect():
        w = b.want
        w.reserve([0, 1, 2, 3], [1] * 4)
        for s in range(4):
            p = w.kv_len[s] - 1
            for c in w.caches:
                c[w.tables[s][p // B], p % B] = 1
        w.free([0, 1, 2, 3], [16] * 4, [n - 24 for n in w.kv_len])
        w.compact()

    step()
    expect()
    b.check(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(40):
        graph.replay()
        expect()
        if turn % 8 == 0:
            b.check(0)
            step()   # an eager one between the replays
            expect()
    b.check(0)


def test_serving_loop():
    """Prompts in chunks, continuations that share them, decoding through a window
    whose passed pages are given back, a compaction on the way: every step's rows
    against the oracle's attention of each sequence's own history."""
    Hq, Hkv, W, sink = 8, 2, 90, 5
    b = Both(8, 40, 150, n_caches=2, Hkv=Hkv, seed=7)
    kv = cp.PagedKV(b.caches[0], b.caches[1], b.tables, b.kv_len)
    g = torch.Generator().manual_seed(8)
    hist = {s: (np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))) for s in range(8)}
    ws = torch.empty(cp.attn_paged_workspace_size(kv, 2000, 400, Hq), dtype=torch.uint8, device=DEV)

    def step(adds, window):
        cp.kv_reserve(b.pool, i32(list(adds)), i32(list(adds.values())), b.missing)
        assert b.missing.tolist() == [0]
        new = [adds.get(s, 0) for s in range(8)]
        start = np.concatenate([[0], np.cumsum(new)])
        q, k, v = randn(g, start[-1], Hq, D), randn(g, start[-1], Hkv, D), randn(g, start[-1], Hkv, D)
        cp.kv_append(kv, k.to(DEV), v.to(DEV), q_start=i32(start))
        o, lse = torch.empty(len(q), Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(len(q), Hq, device=DEV)
        cp.attn_paged(kv, q.to(DEV), o, ws, lse=lse, q_start=i32(start), max_q=max(new), window=window, n_sink=sink)
        lens = b.kv_len.tolist()
        for s in range(8):
            a, e = start[s], start[s + 1]
            hist[s] = tuple(np.concatenate([h, f64(x[a:e])]) for h, x in zip(hist[s], (k, v)))
            assert lens[s] == len(hist[s][0])
            pick = np.unique(np.linspace(0, e - a - 1, 9).astype(int)) if e > a else []
            if len(pick):
                want = owin.attend(f64(q[a:e])[pick], lens[s] - (e - a) + pick, *hist[s], np.arange(lens[s]), window, sink)
                compare(f64(o)[a:e][pick], f64(lse)[a:e][pick], want, lens[s], f"sequence {s}")

    def free_passed(seqs):
        lens = b.kv_len.tolist()
        cp.kv_free(b.pool, i32(seqs), i32([sink] * len(seqs)), i32([max(0, lens[s] - W) for s in seqs]))

    step({0: 130, 1: 47, 2: 333}, 0)
    step({0: 50, 1: 1, 2: 17}, 0)
    cp.kv_fork(b.pool, i32([0, 0, 2]), i32([3, 4, 5]), b.missing)
    for a, c in ((0, 3), (0, 4), (2, 5)):
        hist[c] = hist[a]
    for turn in range(12):
        step({s: 1 for s in range(6)}, W)
        free_passed([0, 1, 2, 3, 4, 5])
        if turn % 4 == 2:
            cp.kv_compact(b.pool, ws)
    used = int((b.refs > 0).sum())
    cp.kv_free(b.pool, i32([2, 5]), i32([0, 0]), i32([10**6, 10**6]))
    assert int((b.refs > 0).sum()) < used and b.kv_len.tolist()[2] == 0
    hist[2] = hist[5] = (np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D)))
    step({2: 200, 3: 4, 0: 1}, W)
    count = torch.zeros_like(b.refs).index_add_(0, b.tables[b.tables >= 0].long(), torch.ones_like(b.tables[b.tables >= 0]))
    assert torch.equal(count, b.refs)


def test_reserve_where_the_last_page_is_gone():
    """A sequence whose last page, filled in part, was given back: more tokens have no
    place in it.  The entry is missing and changes nothing; one that adds nothing, one
    whose length ends on a page and the other entries of the list are served."""
    b = Both(5, 8, 40, seed=10)
    b.reserve([0, 1, 2, 3], [37, 32, 45, 20])
    b.free([0, 1, 2], [5, 16, 32], [37, 32, 45])      # their last pages, the lengths stay
    b.reserve([0, 1, 2, 3], [1, 1, 40, 1])
    assert b.missing.tolist() == [2] and b.kv_len.tolist() == [37, 33, 45, 21, 0]
    b.reserve([0, 2], [0, 0])
    assert b.missing.tolist() == [0]
    b.tables[3, 1], b.want.tables[3][1] = 40, 40      # no page of the pool either
    cp.kv_reserve(b.pool, i32([3]), i32([1]), b.missing)
    assert b.missing.tolist() == [1] and b.want.reserve([3], [1]) == 1 and b.kv_len.tolist() == b.want.kv_len


def test_tokens_reserved_are_tokens_kept():
    """Free, reserve, append, attend: what reserve says it has served is in the cache."""
    Hq, Hkv = 8, 2
    b = Both(3, 8, 40, n_caches=2, Hkv=Hkv, seed=11)
    kv = cp.PagedKV(b.caches[0], b.caches[1], b.tables, b.kv_len)
    g = torch.Generator().manual_seed(12)
    b.reserve([0, 1, 2], [37, 48, 40])
    b.free([0, 1], [5, 32], [37, 48])
    before = b.kv_len.tolist()
    cp.kv_reserve(b.pool, i32([0, 1, 2]), i32([9, 9, 9]), b.missing)
    grown = [n > m for n, m in zip(b.kv_len.tolist(), before)]
    assert b.missing.tolist() == [grown.count(False)]
    k, v = randn(g, 27, Hkv, D), randn(g, 27, Hkv, D)
    cp.kv_append(kv, k.to(DEV), v.to(DEV))
    for s in range(3):
        if grown[s]:
            for i in range(9):
                p = b.kv_len.tolist()[s] - 9 + i
                page = int(b.tables[s, p // B])
                assert page >= 0 and torch.equal(b.caches[0][page, p % B].cpu(), k[9 * s + i])
                assert torch.equal(b.caches[1][page, p % B].cpu(), v[9 * s + i])
    # A window of the appended tokens: attention reads what was appended.
    o, lse = torch.empty(27, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(27, Hq, device=DEV)
    q = randn(g, 27, Hq, D)
    ws = torch.empty(cp.attn_paged_workspace_size(kv, 27, 9, Hq), dtype=torch.uint8, device=DEV)
    cp.attn_paged(kv, q.to(DEV), o, ws, lse=lse, window=9)
    for s in range(3):
        if grown[s]:
            r = slice(9 * s + 8, 9 * s + 9)
            want = owin.attend(f64(q)[r], [8], f64(k)[9 * s:9 * s + 9], f64(v)[9 * s:9 * s + 9], np.arange(9))
            compare(f64(o)[r], f64(lse)[r], want, 9, f"sequence {s}")


def test_fork_where_the_last_page_is_gone():
    """A parent whose last page, filled in part, was given back: there is nothing to
    copy, so its child gets nothing and is missing.  Pages gone before it, or a length
    that ends on a page, are shared as they are."""
    b = Both(9, 8, 40, n_caches=2, seed=13)
    b.reserve([0, 1, 2, 3], [37, 48, 45, 70])
    b.free([0, 1, 3], [5, 32, 16], [37, 48, 64])
    b.fork([0, 1, 2, 3, 0], [4, 5, 6, 7, 8])
    assert b.missing.tolist() == [2] and b.kv_len.tolist()[4:] == [0, 48, 45, 70, 0]
    b.reserve([5, 6, 7], [3, 3, 3])                   # what was served can go on
    assert b.missing.tolist() == [0]


def test_caches_of_one_tensor():
    """A pool's caches as the slices of one tensor, or from an iterator."""
    pair = torch.zeros(2, 12, B, 2, D, dtype=torch.bfloat16, device=DEV)
    pair[:, 0] = 7
    tables, kv_len, refs = torch.full((2, 4), -1, dtype=torch.int32, device=DEV), i32([5, 0]), i32([1] + [0] * 11)
    tables[0, 0] = 0
    missing = i32([-1])
    for caches in (pair, iter(pair), iter([])):
        pool = cp.KVPool(tables, kv_len, refs, caches)
        cp.kv_fork(pool, i32([0]), i32([1]), missing)
        assert missing.tolist() == [0] and tables[1].tolist() == [1, -1, -1, -1]
        cp.kv_free(pool, i32([1]), i32([0]), i32([5]))
    assert (pair[:, 1] == 7).all()
