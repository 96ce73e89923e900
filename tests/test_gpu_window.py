"""GPU checks of cp_attn_window, a rank's zigzag rows through a sliding window,
against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import window as owin
from oracle.attention import gather_paged
from paper_2609_04774_amd import cpattn as cp

from paged_cases import B, D, DEV, compare, f64, randn

pytestmark = pytest.mark.gpu


def run(P, R, C, Hq, Hkv, window, n_sink, seed, order=cp.CP_OUT_LOCAL, edit=None, rows_checked=None, scale=0.0):
    """Every rank's rows against the oracle; returns the outputs of the last rank."""
    g = torch.Generator().manual_seed(seed)
    q, k, v = randn(g, R, Hq, D), randn(g, R, Hkv, D), randn(g, R, Hkv, D)
    n_blocks = P // B + 3
    kc, vc = randn(g, n_blocks, B, Hkv, D), randn(g, n_blocks, B, Hkv, D)
    table = torch.randperm(n_blocks, generator=g)[:P // B].to(torch.int32)
    if edit:
        edit(k, v, kc, vc, table)
    dev = [t.to(DEV) for t in (q, k, v, kc, vc, table)]
    keys = np.concatenate([gather_paged(f64(kc), table.numpy(), P), f64(k)])
    vals = np.concatenate([gather_paged(f64(vc), table.numpy(), P), f64(v)])
    out = None
    for r in range(C):
        plan, rows = cp.shard_plan(P, R, C, r)
        if plan.n_rows == 0:
            continue
        qr = dev[0][torch.as_tensor(rows - P, device=DEV)].contiguous()
        n_out = R if order == cp.CP_OUT_SEQUENCE else plan.n_rows
        o = torch.full((n_out, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        lse = torch.full((n_out, Hq), float("nan"), device=DEV)
        ws = torch.empty(cp.attn_window_workspace_size(plan, Hq, Hkv), dtype=torch.uint8, device=DEV)
        cp.attn_window(plan, qr, dev[1], dev[2], o, ws, window, n_sink=n_sink, lse=lse, k_cache=dev[3], v_cache=dev[4],
                       block_table=dev[5], out_order=order, softmax_scale=scale)
        if order == cp.CP_OUT_SEQUENCE:
            mine = np.zeros(R, bool)
            mine[rows - P] = True
            assert torch.isnan(lse[torch.as_tensor(~mine, device=DEV)]).all()  # other ranks' rows
            at = rows - P
        else:
            at = np.arange(plan.n_rows)
        pick = np.arange(plan.n_rows) if rows_checked is None else np.unique(np.clip(rows_checked, 0, plan.n_rows - 1))
        want = owin.attend(f64(q)[rows[pick] - P], rows[pick], keys, vals, np.arange(P + R), window, n_sink,
                           scale or None)
        compare(f64(o)[at[pick]], f64(lse)[at[pick]], want, P + R, f"rank {r}")
        out = o, lse, rows
    return out


@pytest.mark.parametrize("P,R,C", [(0, 1, 1), (0, 37, 2), (16, 5, 4), (64, 300, 1), (160, 333, 2), (48, 515, 3)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (17, 3), (64, 20), (1000, 4)])
def test_shapes(P, R, C, window, n_sink):
    run(P, R, C, 8, 2, window, n_sink, seed=P + R + C + window, rows_checked=np.arange(0, 600, 11))


@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 1), (28, 4), (64, 8)])
def test_heads_and_sequence_order(Hq, Hkv):
    run(96, 200, 2, Hq, Hkv, 70, 5, seed=7, order=cp.CP_OUT_SEQUENCE, rows_checked=np.arange(0, 200, 17))


def test_scale():
    run(32, 100, 1, 8, 2, 40, 2, seed=8, scale=0.21)


def test_without_a_window():
    """Window 0: every key before a row, for every rank."""
    run(128, 700, 4, 8, 2, 0, 0, seed=9, rows_checked=np.arange(0, 200, 7))


def test_long_window():
    run(4096, 4100, 2, 8, 1, 3000, 9, seed=10, rows_checked=np.array([0, 1, 500, 1023, 1024, 1025, 2040, 2049]))


def test_many_rows_in_sequence_order():
    """Enough rows for wide blocks, over the prefix and the new tokens."""
    run(4800, 16384, 2, 16, 1, 0, 0, seed=14, order=cp.CP_OUT_SEQUENCE,
        rows_checked=np.array([0, 95, 96, 255, 256, 4095, 4096, 8191]))


def test_pages_that_name_nothing():
    def edit(k, v, kc, vc, table):
        table[2], table[4] = -1, len(kc)
    run(96, 60, 2, 8, 2, 50, 40, seed=11, edit=edit)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_keys_outside_every_window(bad):
    """What lies between the first tokens and the first row's window has no part in
    any row."""
    def edit(k, v, kc, vc, table):
        for j in range(6, 96 - 40):
            kc[table[j // B], j % B] = bad
            vc[table[j // B], j % B] = bad
    g = run(96, 100, 1, 8, 2, 40, 6, seed=12)
    h = run(96, 100, 1, 8, 2, 40, 6, seed=12, edit=edit)
    assert torch.equal(g[0], h[0]) and torch.equal(g[1], h[1])


def test_later_values_do_not_reach_earlier_rows():
    clean = run(0, 300, 1, 8, 2, 64, 4, seed=13)

    def edit(k, v, kc, vc, table):
        v[150, 0, 7] = float("nan")
        v[200, 1, 3] = float("inf")
    g = torch.Generator().manual_seed(13)
    q, k, v = randn(g, 300, 8, D), randn(g, 300, 2, D), randn(g, 300, 2, D)
    edit(k, v, None, None, None)
    plan, _ = cp.shard_plan(0, 300, 1, 0)
    o = torch.empty(300, 8, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(cp.attn_window_workspace_size(plan, 8, 2), dtype=torch.uint8, device=DEV)
    cp.attn_window(plan, q.to(DEV), k.to(DEV), v.to(DEV), o, ws, 64, n_sink=4)
    got, want = f64(o), f64(clean[0])
    hit = np.zeros_like(got, bool)
    hit[150:214, :4, 7] = True
    hit[200:264, 4:, 3] = True
    assert np.isnan(got[150:214, :4, 7]).all() and np.isposinf(got[200:264, 4:, 3]).all()
    assert np.isfinite(got[~hit]).all()
    assert np.abs(got - want)[~hit].max() <= 2.0**-7 * np.abs(want).max()


def test_prefix_offsets_beyond_32_bits():
    P, R = 64, 70
    g = torch.Generator().manual_seed(15)
    q, k, v, pk, pv = (randn(g, n, h, D) for n, h in ((R, 32), (R, 8), (R, 8), (P, 8), (P, 8)))
    kc = torch.empty(140000, B, 8, D, dtype=torch.bfloat16, device=DEV)  # 4.6 GB
    vc = torch.empty_like(kc)
    table = torch.tensor([139999, 139000, 5, 139500], dtype=torch.int32, device=DEV)
    kc[table.long()], vc[table.long()] = pk.view(4, B, 8, D).to(DEV), pv.view(4, B, 8, D).to(DEV)
    plan, rows = cp.shard_plan(P, R, 1, 0)
    o, lse = torch.empty(R, 32, D, dtype=torch.bfloat16, device=DEV), torch.empty(R, 32, device=DEV)
    ws = torch.empty(cp.attn_window_workspace_size(plan, 32, 8), dtype=torch.uint8, device=DEV)
    cp.attn_window(plan, q.to(DEV), k.to(DEV), v.to(DEV), o, ws, 50, n_sink=3, lse=lse, k_cache=kc, v_cache=vc,
                   block_table=table)
    want = owin.attend(f64(q), rows, np.concatenate([f64(pk), f64(k)]), np.concatenate([f64(pv), f64(v)]),
                       np.arange(P + R), 50, 3)
    compare(f64(o), f64(lse), want, P + R, "rows")


def test_plan_without_rows():
    plan, _ = cp.shard_plan(0, 3, 8, 5)
    assert plan.n_rows == 0
    t = torch.empty(3, 2, D, dtype=torch.bfloat16, device=DEV)
    cp.attn_window(plan, t[:0].repeat(1, 4, 1), t, t, t[:0].repeat(1, 4, 1), torch.empty(256, dtype=torch.uint8, device=DEV), 4)
