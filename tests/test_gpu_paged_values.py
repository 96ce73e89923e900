"""GPU checks of what cp_attn_paged and cp_attn_window make of particular values:
O as a mean of the values with the weights that were used, and infinite or NaN
values of keys whose weight is nothing."""

import numpy as np
import pytest
import torch

from paper_2609_04774_amd import cpattn as cp

from paged_cases import D, DEV, Batch, randn

pytestmark = pytest.mark.gpu

TILES = {128: 0, 256: 1, 384: 2}


def refill(b):
    starts = torch.tensor(np.concatenate([[0], np.cumsum(b.kv_len)]), dtype=torch.int32, device=DEV)
    cp.kv_append(b.kv, torch.cat(b.k).to(DEV), torch.cat(b.v).to(DEV), q_start=starts)


def run(b, rows=None, **args):
    """A launch; with `rows`, one whose lengths choose blocks of so many rows (the
    workspace says which, behind the 256 shares' starts)."""
    ws = torch.empty(cp.attn_paged_workspace_size(b.kv, len(b.q), b.max_q, b.Hq), dtype=torch.uint8, device=DEV)
    out = b.run(ws=ws, **args)
    if rows is not None:
        assert ws.view(torch.int32)[1024] == TILES[rows]
    return out


# (lengths, rows of each, query heads, KV heads, rows of a block or None for few rows)
SHAPES = [
    ([1, 17, 300, 2048, 4096], [1] * 5, 8, 2, None),
    ([60, 1000, 4096, 33], [7] * 4, 8, 2, None),
    ([777] * 5, [100] * 5, 2, 2, 128),
    ([4096], [64], 8, 1, 128),
    ([1500, 1400, 1600, 1211, 50, 1550, 850, 1400], [250, 256, 255, 300, 0, 512, 1, 256], 64, 64, 256),
    ([4096] * 16, [1536] * 16, 16, 1, 384),
]


def constant(b, g):
    """Every key's value is its sequence's and head's: the mean of any weights."""
    for s, t in enumerate(b.kv_len):
        # From 255 / 128 on the next bf16 value is nearest, relative to the value: 2^-8.
        v = randn(g, b.k[s].shape[1], D)
        v[:, ::2] = 255 / 128
        b.v[s] = v.expand(t, -1, -1).contiguous()


def check_constant(b, o):
    """Bit by bit.  Of n keys O is sum p v / sum p with the same weights p above and
    below: products exact, sums of one sign within n 2^-24 each, at most as many
    rescalings of a running maximum, 64 more roundings where parts are joined: 2 (2 n +
    64) 2^-24 < 2^-10 of v for n <= 4096, and half of a bf16 step is 2^-9 or more."""
    assert max(b.kv_len) <= 4096
    heads = torch.arange(b.Hq) // (b.Hq // b.k[0].shape[1])
    for s, t in enumerate(b.kv_len):
        if b.new[s]:
            got = o[b.start[s]:b.start[s + 1]]
            assert torch.equal(got, b.v[s][0, heads].to(DEV).expand(len(got), -1, -1)), f"sequence {s} ({t} positions)"


@pytest.mark.parametrize("lens,new,Hq,Hkv,rows", SHAPES)
def test_mean_of_equal_values(lens, new, Hq, Hkv, rows):
    """Random scores, with and without a window."""
    b = Batch(lens, new, Hq, Hkv, seed=101, uniform=len(set(new)) == 1)
    constant(b, torch.Generator().manual_seed(102))
    refill(b)
    check_constant(b, run(b, rows)[0])
    check_constant(b, b.run(700, 9)[0])


@pytest.mark.parametrize("lens,new,Hq,Hkv,rows", SHAPES)
def test_mean_of_equal_values_of_one_weight(lens, new, Hq, Hkv, rows):
    """All keys but the first weigh e^-0.6895 = 0.5018 of its weight, which bf16 holds
    as 0.5: the roundings have one sign."""
    b = Batch(lens, new, Hq, Hkv, seed=103, uniform=len(set(new)) == 1)
    constant(b, torch.Generator().manual_seed(104))
    b.q.zero_()
    b.q[:, :, 0] = b.q[:, :, 1] = 1
    for k in b.k:
        k.zero_()
        k[:1, :, 0], k[:1, :, 1] = 0.6875, 0.002
    refill(b)
    o, lse = run(b, rows, scale=1.0)
    check_constant(b, o)
    for s, t in enumerate(b.kv_len):
        if b.new[s]:  # the LSE's sum is of the weights before their rounding
            n = torch.arange(t - b.new[s], t, device=DEV, dtype=torch.float64)[:, None]
            x = float(b.k[s][0, 0, 0]) + float(b.k[s][0, 0, 1])
            want = torch.log(np.exp(x) + n)
            assert (lse[b.start[s]:b.start[s + 1]] - want).abs().max() < 1e-4


def test_mean_of_equal_values_of_a_rank():
    P, R, Hq, Hkv = 640, 1500, 8, 2
    g = torch.Generator().manual_seed(105)
    v = randn(g, Hkv, D)
    v[:, ::2] = 255 / 128
    q, k = randn(g, R, Hq, D).to(DEV), randn(g, R, Hkv, D).to(DEV)
    kc = randn(g, P // 16, 16, Hkv, D).to(DEV)
    vc = v.expand(P // 16, 16, Hkv, D).contiguous().to(DEV)
    vn = v.expand(R, Hkv, D).contiguous().to(DEV)
    table = torch.arange(P // 16, dtype=torch.int32, device=DEV)
    plan, rows = cp.shard_plan(P, R, 2, 1)
    ws = torch.empty(cp.attn_window_workspace_size(plan, Hq, Hkv), dtype=torch.uint8, device=DEV)
    for window in (0, 300):
        o = torch.zeros(plan.n_rows, Hq, D, dtype=torch.bfloat16, device=DEV)
        cp.attn_window(plan, q[torch.as_tensor(rows - P, device=DEV)].contiguous(), k, vn, o, ws, window, n_sink=5,
                       k_cache=kc, v_cache=vc, block_table=table)
        assert torch.equal(o, v[torch.arange(Hq) // 4].to(DEV).expand_as(o))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("lens,new,Hq,Hkv,rows", [
    ([700], [1], 8, 2, None), ([700], [5], 8, 2, None), ([700], [100], 2, 2, 128),
    ([1400, 1500, 1600, 1550], [512] * 4, 64, 64, 256), ([2048] * 40, [1024] * 40, 16, 1, 384),
])
def test_values_of_weight_nothing(lens, new, Hq, Hkv, rows, bad):
    """A key that a row sees, e^-200 below the others (in fp32 its weight is 0): an
    infinity or NaN among its values shows in the row, wherever the key lies -- behind
    other keys or before them, in a tile that every row sees or at the mask's edge, in
    a part of its own -- and in no row that does not see it."""
    b = Batch(lens, new, Hq, Hkv, seed=106, uniform=True)
    b.q.zero_()
    b.q[:, :, 0] = 1
    n = new[0]
    for at in (0, 40, 333, lens[0] - n, lens[0] - n // 2 - 1, lens[0] - 1):
        for whole in (False, True):  # the key alone, or all those around it
            for k, v in zip(b.k, b.v):
                k.zero_()
                v.fill_(1)
                k[max(0, at - 100 * whole):at + 1, :, 0] = -200
                v[at, 0, 3] = bad
            refill(b)
            o, _ = run(b, rows, scale=1.0)
            o = o.view(len(lens), n, Hq, D).float()
            for s, t in enumerate(lens):
                sees = torch.arange(t - n, t, device=DEV) >= at
                shown = ~torch.isfinite(o[s])
                hit = torch.zeros_like(shown)
                hit[sees, :Hq // Hkv, 3] = True
                assert torch.equal(shown, hit), (at, whole, s)
