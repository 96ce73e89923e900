"""GPU checks of cp_attn_paged (single tokens, chunks, mixed batches; windows) and
cp_kv_append against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import window as owin
from paper_2609_04774_amd import cpattn as cp

from paged_cases import B, D, DEV, Batch, compare, f64, randn

pytestmark = pytest.mark.gpu

HEADS = [(8, 2), (4, 4), (8, 1), (28, 4), (64, 8)]


@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("new", [1, 2, 5])
def test_decode_lengths(Hq, Hkv, new):
    """Lengths around tile, page and step borders, none and one among them."""
    lens = [0, 1, 5, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 1111]
    b = Batch(lens, [new] * len(lens), Hq, Hkv, seed=10 + new, uniform=True)
    b.check(*b.run())


@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (16, 0), (33, 4), (100, 16), (100, 40), (127, 33), (5000, 7)])
@pytest.mark.parametrize("new", [1, 3])
def test_decode_window(window, n_sink, new):
    lens = [0, 1, 16, 33, 100, 133, 161, 500, 777]
    b = Batch(lens, [new] * len(lens), 8, 2, seed=30 + window, uniform=True)
    b.hide(window, n_sink)
    b.check(*b.run(window, n_sink), window, n_sink)


@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_ragged_chunks(Hq, Hkv):
    """Chunks behind contexts of any length, sequences without rows, one token
    and long chunks in one launch."""
    new = [7, 0, 1, 130, 33, 64, 300, 1]
    lens = [7, 90, 1, 131, 77, 400, 300, 640]
    b = Batch(lens, new, Hq, Hkv, seed=50)
    b.check(*b.run(), rows=np.array([0, 1, 15, 16, 31, 32, 63, 64, 129, 255, 256, 10**6]))


@pytest.mark.parametrize("window,n_sink", [(1, 0), (20, 3), (64, 0), (200, 40), (1000, 5)])
def test_chunk_window(window, n_sink):
    new, lens = [257, 3, 90, 40], [600, 700, 90, 300]
    b = Batch(lens, new, 8, 2, seed=60)
    b.hide(window, n_sink)
    b.check(*b.run(window, n_sink), window, n_sink, rows=np.arange(0, 300, 13))


def test_one_long_sequence():
    """Many shares of one walk, and their merge."""
    b = Batch([20011], [1], 8, 2, seed=70, uniform=True)
    b.check(*b.run())


def test_more_sequences_than_threads():
    rng = np.random.RandomState(5)
    lens = rng.randint(0, 60, 700).tolist()
    new = [min(int(x), t) for x, t in zip(rng.randint(0, 4, 700), lens)]
    b = Batch(lens, new, 4, 2, seed=71)
    b.check(*b.run())


def test_rows_before_the_first_position():
    """More new rows than positions: those below position 0 see no key."""
    b = Batch([3, 0, 20], [5, 5, 5], 8, 2, seed=72, uniform=True)
    o, lse = b.run()
    assert (o[:2] == 0).all() and torch.isneginf(lse[:2]).all()
    assert (o[5:10] == 0).all() and torch.isneginf(lse[5:10]).all()
    b.check(o, lse)


def test_rows_outside_the_sequences_are_left():
    b = Batch([40, 50], [3, 4], 8, 2, seed=73)
    b.q = torch.cat([b.q, b.q[:4]])
    o, lse = b.run()
    assert torch.isnan(o[7:]).all() and torch.isnan(lse[7:]).all()
    b.check(o[:7], lse[:7])
    b.q = b.q[:7]
    b.max_q = 2  # rows past it are left too
    o, _ = b.run()
    assert not torch.isnan(o[[0, 1, 3, 4]]).any() and torch.isnan(o[[2, 5, 6]]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new", [4, 100])
def test_values_that_a_row_does_not_see(bad, new):
    """A later token's K and V, infinite or NaN, change nothing for the rows before
    it; the rows that see them show them."""
    b = Batch([200], [new], 8, 2, seed=74)
    at = 200 - new // 2
    page, slot = int(b.tables[0, at // B]), at % B
    b.vc[page, slot, 1, 5] = bad
    b.v[0][at, 1, 5] = bad
    o, lse = b.run()
    want = f64(o)
    early = new - new // 2
    assert np.isfinite(want[:early]).all()
    seen = want[early:, 4:, 5]
    assert np.isnan(seen).all() if np.isnan(bad) else (seen == bad).all()
    assert np.isfinite(np.delete(want[early:], 5, axis=2)).all() and np.isfinite(want[early:, :4]).all()
    b.v[0][at, 1, 5] = 0.0
    keep = b.new
    res = owin.attend(f64(b.q)[:early], b.positions(0)[:early], f64(b.k[0]), f64(b.v[0]), np.arange(200))
    compare(want[:early], f64(lse)[:early], res, 200, "rows before")
    assert keep == b.new
    b.kc[page, slot, 1] = float("nan")
    o, lse = b.run()
    compare(f64(o)[:early], f64(lse)[:early], res, 200, "rows before, K")
    assert torch.isnan(o[early:, 4:]).all() and torch.isneginf(lse[early:, 4:]).all()


def test_pages_that_name_nothing_read_as_zeros():
    b = Batch([100, 64], [1, 1], 8, 2, seed=75, uniform=True)
    b.tables[0, 1], b.tables[0, 3], b.tables[1, 0] = -1, b.n_blocks, 2**31 - 1
    b.dev_tables.copy_(b.tables)
    for s, p in ((0, 1), (0, 3), (1, 0)):
        b.k[s][16 * p:16 * p + 16] = 0
        b.v[s][16 * p:16 * p + 16] = 0
    b.check(*b.run())


@pytest.mark.parametrize("new", [1, 4, 60])
def test_positions_beyond_the_table_have_no_keys(new):
    """A length that its table does not cover: the rows at its end see what the
    table holds (an odd number of pages: half a tile)."""
    b = Batch([80, 40], [new, new], 8, 2, seed=76, uniform=True, table_extra=0)
    o, lse = torch.empty(2 * new, 8, D, dtype=torch.bfloat16, device=DEV), torch.empty(2 * new, 8, device=DEV)
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, 2 * new, new, 8), dtype=torch.uint8, device=DEV)
    for length in (100, 2**31 - 1):
        for window, n_sink in ((0, 0), (120, 3), (33, 20)):
            b.dev_len[0] = length
            cp.attn_paged(b.kv, b.q.to(DEV), o, ws, lse=lse, window=window, n_sink=n_sink)
            pos = min(length, 2**30) - new + np.arange(new)
            want = owin.attend(f64(b.q)[:new], pos, f64(b.k[0]), f64(b.v[0]), np.arange(80), window, n_sink)
            compare(f64(o)[:new], f64(lse)[:new], want, 80, f"length {length}, window {window}")
            want = owin.attend(f64(b.q)[new:], b.positions(1), f64(b.k[1]), f64(b.v[1]), np.arange(40), window, n_sink)
            compare(f64(o)[new:], f64(lse)[new:], want, 40, "the other sequence")


def test_a_long_chunk_among_many_sequences():
    """Most sequences have one row, one has many, some none, in any order."""
    rng = np.random.RandomState(6)
    new = [1] * 300
    new[7], new[150], new[299] = 700, 0, 40
    lens = [n + int(x) for n, x in zip(new, rng.randint(0, 90, 300))]
    b = Batch(lens, new, 8, 1, seed=82)
    b.check(*b.run(), rows=np.array([0, 1, 31, 32, 300, 699]))
    b.check(*b.run(50, 4), 50, 4, rows=np.array([0, 1, 31, 32, 300, 699]))


def blocks_of(rows, b, window=0, n_sink=0):
    """A launch whose lengths choose blocks of so many rows (the workspace says which,
    behind the 256 shares' starts)."""
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, len(b.q), b.max_q, b.Hq), dtype=torch.uint8, device=DEV)
    out = b.run(window, n_sink, ws=ws)
    assert ws.view(torch.int32)[1024] == [128, 256, 384].index(rows)
    return out


def wide(b, window=0, n_sink=0):
    return blocks_of(384, b, window, n_sink)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1000, 0), (1100, 40)])
def test_blocks_of_256_rows(window, n_sink):
    b = Batch([1500, 1400, 1600, 1211, 50, 1550, 850, 1400], [250, 256, 255, 300, 0, 512, 1, 256], 64, 64, seed=91)
    rows = np.array([0, 1, 31, 32, 100, 127, 128, 200, 249, 255, 256, 299, 511])
    if window:
        b.hide(window, n_sink)
    b.check(*blocks_of(256, b, window, n_sink), window, n_sink, rows=rows)


@pytest.mark.parametrize("rows,heads,new", [(128, 2, 100), (256, 64, 256)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_in_blocks(rows, heads, new, bad):
    """As above, in blocks of many rows: an infinite or NaN value of one head."""
    n = 5
    b = Batch([777] * n, [new] * n, heads, heads, seed=92, uniform=True)
    for s in range(n):
        b.v[s][777 - new // 2, 1, 9] = bad
    starts = torch.arange(0, 777 * n + 1, 777, dtype=torch.int32, device=DEV)
    cp.kv_append(b.kv, torch.cat(b.k).to(DEV), torch.cat(b.v).to(DEV), q_start=starts)
    o, lse = blocks_of(rows, b)
    got = o.float().view(n, new, heads, D)
    seen = got[:, new - new // 2:, 1, 9]
    assert torch.isnan(seen).all() if np.isnan(bad) else (seen == bad).all()
    finite = torch.isfinite(got)
    finite[:, new - new // 2:, 1, 9] = True
    assert finite.all()
    b.check(o, lse, rows=np.array([0, 1, new // 2 - 1, new // 2, new - new // 2 - 1, new - new // 2, new - 1]))


def test_wide_blocks():
    b = Batch([17300, 40, 9000], [8192, 3, 129], 16, 1, seed=83)
    rows = np.array([0, 1, 23, 24, 95, 96, 128, 383, 384, 1000, 4097, 8190, 8191])
    first = wide(b)
    b.check(*first, rows=rows)
    again = wide(b)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    # A later token's infinite value shows in the rows that see it, in its column.  (The
    # others keep their results within the bounds, not their bits: such a tile is taken
    # by itself, and the weights around it against another maximum.)
    at = 17300 - 4000
    page, slot = int(b.tables[0, at // B]), at % B
    b.vc[page, slot, 0, 7] = float("inf")
    o, lse = wide(b)
    i = 8192 - 4000
    assert torch.equal(lse[8192:], first[1][8192:]) and torch.equal(o[8192:], first[0][8192:])
    finite = torch.isfinite(o[:8192].float())
    assert finite[:i].all() and not finite[i:, :, 7].any()
    finite[:, :, 7] = True
    assert finite.all()
    b.v[0][at, 0, 7] = float("inf")
    b.check(o, lse, rows=rows)


def test_wide_blocks_window():
    b = Batch([30000], [12288], 16, 1, seed=84)
    b.hide(16384, 5)
    b.check(*wide(b, 16384, 5), 16384, 5, rows=np.array([0, 95, 96, 1000, 5555, 12287]))


def test_captured_launch_follows_the_choice_of_blocks():
    """Replays of one capture whose lengths ask for wide blocks, for narrow ones, and
    for wide ones again, against the oracle and the eager call."""
    b = Batch([17300], [8192], 16, 1, seed=85)
    rows = np.array([0, 95, 96, 255, 256, 4097, 8191])
    q = b.q.to(DEV)
    o, lse = torch.empty_like(q), torch.empty(8192, 16, device=DEV)
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, 8192, 8192, 16), dtype=torch.uint8, device=DEV)

    def step():
        cp.attn_paged(b.kv, q, o, ws, lse=lse, q_start=b.q_start, max_q=8192)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for length, is_wide in ((17300, True), (8192, False), (5000, False), (17300, True)):
        b.kv_len[0] = length
        b.dev_len.fill_(length)
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert (ws.view(torch.int32)[1024] == 2) == is_wide
        got = o.clone(), lse.clone()
        k, v = b.k[0], b.v[0]
        b.k[0], b.v[0] = k[:length], v[:length]
        b.check(*got, rows=rows)
        b.k[0], b.v[0] = k, v
        step()
        assert torch.equal(o, got[0]) and torch.equal(lse, got[1])


def test_scale_and_strided_queries():
    b = Batch([77, 200, 9], [2, 2, 2], 8, 2, seed=77, uniform=True)
    o, lse = b.run(scale=0.3)
    b.check(o, lse, scale=0.3)
    wide = torch.full((6, 8 + 4, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :8] = b.q.to(DEV)
    got = torch.empty(6, 8, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, 6, 2, 8), dtype=torch.uint8, device=DEV)
    cp.attn_paged(b.kv, wide[:, :8], got, ws, softmax_scale=0.3)  # no LSE
    assert torch.equal(got, o)


def test_large_scores_and_sinks():
    """First tokens of far larger scores, and scores over a wide range."""
    b = Batch([700], [3], 8, 2, seed=78, uniform=True)
    b.k[0][:4] *= 12
    b.k[0][100:] *= 4
    starts = torch.tensor([0, 700], dtype=torch.int32, device=DEV)
    cp.kv_append(b.kv, b.k[0].to(DEV), b.v[0].to(DEV), q_start=starts)
    b.check(*b.run())
    b.check(*b.run(64, 4), 64, 4)


def test_repeated_calls_agree():
    b = Batch([5000, 3, 900, 2500], [1, 1, 1, 1], 32, 8, seed=79, uniform=True)
    first = b.run()
    for _ in range(3):
        again = b.run()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_captured_launch_follows_the_lengths():
    """One captured step (append, attend), replayed while lengths, tables and rows
    change, against the eager calls."""
    Hq, Hkv, n = 8, 2, 5
    b = Batch([40, 1, 300, 17, 64], [1] * n, Hq, Hkv, seed=80, uniform=True, spare=200, table_extra=80)
    free = [p for p in range(b.n_blocks) if p not in set(b.tables.flatten().tolist())]
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.empty(n, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    o, lse = torch.empty(n, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, Hq, device=DEV)
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, n, 1, Hq), dtype=torch.uint8, device=DEV)

    def step():
        cp.kv_append(b.kv, k, v)
        cp.attn_paged(b.kv, q, o, ws, lse=lse)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q.copy_(b.q.to(DEV)), k.zero_(), v.zero_()
        step()  # (position kv_len - 1 is written again below)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn, add in enumerate([0, 1, 1, 40, 200]):
        for s in range(n):
            old, b.kv_len[s] = b.kv_len[s], b.kv_len[s] + add
            b.k[s], b.v[s] = (torch.cat([x, randn(g, add, Hkv, D)]) for x in (b.k[s], b.v[s]))
            for j in range(-(-old // B), -(-b.kv_len[s] // B)):
                b.tables[s, j] = free.pop()
        b.dev_tables.copy_(b.tables)
        b.dev_len.copy_(torch.tensor(b.kv_len, dtype=torch.int32))
        starts = torch.tensor(np.concatenate([[0], np.cumsum(b.kv_len)]), dtype=torch.int32, device=DEV)
        cp.kv_append(b.kv, torch.cat(b.k).to(DEV), torch.cat(b.v).to(DEV), q_start=starts)
        b.q = randn(g, n, Hq, D)
        q.copy_(b.q.to(DEV))
        k.copy_(torch.stack([x[-1] for x in b.k]).to(DEV))
        v.copy_(torch.stack([x[-1] for x in b.v]).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        b.check(o, lse)
        got = o.clone()
        step()
        assert torch.equal(got, o), turn


def test_another_stream():
    b = Batch([500, 90], [1, 1], 8, 2, seed=81, uniform=True)
    want = b.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = b.run()
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# --- append ------------------------------------------------------------------------------

@pytest.mark.parametrize("new", [1, 3])
def test_shared_prefixes_in_a_large_pool(new):
    """More pages than the Infinity Cache holds: long walks stream, but for the pages
    that another sequence names too."""
    b = Batch([1700, 1500, 1400, 2000, 60, 1300, 1700], [new] * 7, 8, 2, seed=89, uniform=True, spare=17000)
    for s, tokens in ((1, 800), (2, 1392), (4, 48), (6, 16)):
        b.tables[s, :tokens // B] = b.tables[0, :tokens // B]
        b.k[s][:tokens], b.v[s][:tokens] = b.k[0][:tokens], b.v[0][:tokens]
    b.tables[5, 3] = -1
    b.k[5][48:64] = b.v[5][48:64] = 0
    b.dev_tables.copy_(b.tables)
    b.check(*b.run())
    b.check(*b.run(1350, 20), 1350, 20)


def test_many_sequences_in_a_large_pool():
    rng = np.random.RandomState(9)
    lens = rng.randint(1, 40, 602).tolist()
    lens[3], lens[511], lens[512], lens[600] = 1400, 1500, 1600, 1333
    b = Batch(lens, [1] * 602, 4, 2, seed=90, uniform=True, spare=17000)
    b.check(*b.run())


def test_two_calls_at_once():
    """Calls on two streams, each with its workspace, and a page copy beside them."""
    a = Batch([3000, 50, 900], [1, 1, 1], 8, 2, seed=86, uniform=True)
    b = Batch([700, 300], [200, 64], 8, 2, seed=87)
    want = a.run(), b.run()
    torch.cuda.synchronize()
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    got = [[], []]
    for _ in range(8):
        for side, batch, out in zip(sides, (a, b), got):
            with torch.cuda.stream(side):
                out.append(batch.run())
    torch.cuda.synchronize()
    for out, w in zip(got, want):
        assert all(torch.equal(o, w[0]) and torch.equal(l, w[1]) for o, l in out)


@pytest.mark.parametrize("new", [2, 90])
def test_offsets_beyond_32_bits(new):
    """Pages at the end of caches of 4.6 GB."""
    b = Batch([333, 40], [new, 3], 32, 8, seed=88)
    n = 140000
    kc = torch.empty(n, B, 8, D, dtype=torch.bfloat16, device=DEV)
    vc = torch.empty_like(kc)
    tables = torch.where(b.tables >= 0, n - 1 - b.tables, b.tables).to(DEV)
    kv = cp.PagedKV(kc, vc, tables, b.dev_len)
    starts = torch.tensor([0, 333, 373], dtype=torch.int32, device=DEV)
    cp.kv_append(kv, torch.cat(b.k).to(DEV), torch.cat(b.v).to(DEV), q_start=starts)
    o, lse = torch.empty(new + 3, 32, D, dtype=torch.bfloat16, device=DEV), torch.empty(new + 3, 32, device=DEV)
    ws = torch.empty(cp.attn_paged_workspace_size(kv, new + 3, max(new, 3), 32), dtype=torch.uint8, device=DEV)
    for window in (0, 60):
        cp.attn_paged(kv, b.q.to(DEV), o, ws, lse=lse, q_start=b.q_start, max_q=max(new, 3), window=window, n_sink=2)
        b.check(o, lse, window, 2, rows=np.arange(0, 90, 7))
    pages = tables[tables >= 0].flip(0).contiguous()
    low = torch.arange(len(pages), dtype=torch.int32, device=DEV)
    cp.kv_copy_pages([kc, vc], pages, low)
    for c in (kc, vc):
        assert torch.equal(c[:len(pages)].view(torch.int16), c[pages.long()].view(torch.int16))


@pytest.mark.parametrize("Hkv,head_dim", [(1, 128), (2, 128), (8, 128), (3, 40)])
def test_append_positions(Hkv, head_dim):
    """Ragged rows at odd positions, from a strided source; every other slot, and
    rows outside the sequences, are left alone."""
    g = torch.Generator().manual_seed(90 + Hkv)
    kv_len, new = [5, 33, 16, 100, 4], [5, 7, 1, 0, 6]  # the last: two rows below position 0
    tables = torch.randperm(40, generator=g)[:35].to(torch.int32).view(5, 7)
    tables[1, 2] = -1   # position 32 has no page
    start = np.cumsum([2] + new)
    rows = int(start[-1]) + 3
    fused = randn(g, rows, 2 * Hkv + 1, head_dim).to(DEV)
    kc = randn(g, 40, B, Hkv, head_dim).to(DEV)
    vc = randn(g, 40, B, Hkv, head_dim).to(DEV)
    wk, wv = kc.clone(), vc.clone()
    kv = cp.PagedKV(kc, vc, tables.to(DEV), torch.tensor(kv_len, dtype=torch.int32, device=DEV))
    k, v = fused[:, 1:1 + Hkv], fused[:, 1 + Hkv:]
    cp.kv_append(kv, k, v, q_start=torch.tensor(start, dtype=torch.int32, device=DEV))
    for s in range(5):
        for i in range(new[s]):
            pos = kv_len[s] - new[s] + i
            if pos >= 0 and tables[s, pos // B] >= 0:
                wk[tables[s, pos // B], pos % B] = k[start[s] + i]
                wv[tables[s, pos // B], pos % B] = v[start[s] + i]
    assert torch.equal(kc, wk) and torch.equal(vc, wv)


def test_append_of_more_rows_than_a_launch_holds():
    n = (1 << 24) + 1000  # narrow rows: 2^24 of a launch
    pages = -(-n // B)
    kc = torch.zeros(pages, B, 1, 8, dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    tables = torch.arange(pages, dtype=torch.int32, device=DEV).flip(0).contiguous().view(1, pages)
    kv = cp.PagedKV(kc, vc, tables, torch.tensor([n], dtype=torch.int32, device=DEV))
    rows = (torch.arange(n * 8, dtype=torch.int32, device=DEV) % 30011).to(torch.int16).view(torch.bfloat16).view(n, 1, 8)
    cp.kv_append(kv, rows, rows)
    got = kc.flip(0).reshape(-1, 1, 8)[:n].view(torch.int16)
    assert torch.equal(got, rows.view(torch.int16)) and torch.equal(vc.view(torch.int16), kc.view(torch.int16))


def test_append_past_the_table_is_passed_over():
    kc, vc = (torch.zeros(8, B, 2, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kv = cp.PagedKV(kc, vc, torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4),
                    torch.tensor([70, 2**31 - 1], dtype=torch.int32, device=DEV))
    rows = torch.ones(20, 2, D, dtype=torch.bfloat16, device=DEV)
    cp.kv_append(kv, rows, rows)
    want = torch.zeros_like(kc)
    want[3, 12:] = 1  # positions 60 .. 63 of sequence 0
    assert torch.equal(kc, want) and torch.equal(vc, want)


def test_launches_beside_each_other():
    """Many launches of single tokens and of chunks queued on two streams, each with its
    workspace, and page copies on a third, let go together: the results are the bits of
    the calls by themselves."""
    a = Batch([30000, 50, 9000, 17000], [1] * 4, 8, 2, seed=93, uniform=True)
    b = Batch([6000, 900, 3100], [700, 64, 300], 8, 2, seed=94)
    g = torch.Generator().manual_seed(95)
    caches = [torch.randint(-99, 99, (2000, B, 2, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2)]
    copied = [c.clone() for c in caches]
    src = torch.arange(1000, dtype=torch.int32, device=DEV)
    dst = src + 1000
    n = 12
    calls = []
    for x in (a, b):
        q = x.q.to(DEV)
        size = cp.attn_paged_workspace_size(x.kv, len(q), x.max_q, x.Hq)
        out = [(torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)) for _ in range(n)]
        calls.append((x, q, torch.empty(size, dtype=torch.uint8, device=DEV), out, x.run()))
    big = torch.empty(1 << 30, dtype=torch.uint8, device=DEV), torch.empty(1 << 30, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    go = torch.cuda.Event()
    for _ in range(20):  # some milliseconds, in which the launches queue up
        big[0].copy_(big[1])
    go.record()
    sides = [torch.cuda.Stream() for _ in range(3)]
    for side in sides:
        side.wait_event(go)
    for i in range(n):
        for side, (x, q, ws, out, _) in zip(sides, calls):
            cp.attn_paged(x.kv, q, out[i][0], ws, lse=out[i][1], q_start=x.q_start, max_q=x.max_q, stream=side)
        cp.kv_copy_pages(copied, src, dst, stream=sides[2])
    torch.cuda.synchronize()
    for *_, out, want in calls:
        for o, lse in out:
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    for c, w in zip(copied, caches):
        w[1000:] = w[:1000]
        assert torch.equal(c, w)
