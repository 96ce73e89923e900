"""A batch of sequences in a paged cache for the tests of cp_attn_paged and the
calls on pages: caches whose every unused slot is poisoned, filled through
cp_kv_append, and the float64 oracle of its rows."""

from __future__ import annotations

import numpy as np
import torch

from oracle import window as owin
from paper_2609_04774_amd import cpattn as cp

DEV = "cuda"
B = cp.CP_KV_BLOCK_TOKENS
D = cp.CP_HEAD_DIM


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float32).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


class Batch:
    """Sequences of kv_len[s] positions of which the last new[s] are rows of a
    call.  Page tables are random, unused entries -1, and every cache slot that
    holds no token is NaN."""

    def __init__(self, kv_len, new, Hq, Hkv, seed, spare=3, uniform=False, table_extra=2):
        g = torch.Generator().manual_seed(seed)
        self.kv_len, self.new, self.Hq, self.Hkv = list(kv_len), list(new), Hq, Hkv
        n = len(self.kv_len)
        self.k = [randn(g, t, Hkv, D) for t in self.kv_len]
        self.v = [randn(g, t, Hkv, D) for t in self.kv_len]
        self.q = randn(g, sum(self.new), Hq, D)
        pages = [-(-t // B) for t in self.kv_len]
        self.n_blocks = sum(pages) + spare
        perm = torch.randperm(self.n_blocks, generator=g).to(torch.int32)
        self.tables = torch.full((n, max(pages + [0]) + table_extra), -1, dtype=torch.int32)
        at = 0
        for s, m in enumerate(pages):
            self.tables[s, :m] = perm[at:at + m]
            at += m
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.q_start = None if uniform else torch.tensor(self.start, device=DEV)
        self.max_q = max(self.new + [1])
        self.dev_tables = self.tables.to(DEV)
        self.dev_len = torch.tensor(self.kv_len, dtype=torch.int32, device=DEV)
        shape = (self.n_blocks, B, Hkv, D)
        self.kc = torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV)
        self.vc = torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV)
        self.kv = cp.PagedKV(self.kc, self.vc, self.dev_tables, self.dev_len)
        starts = torch.tensor(np.concatenate([[0], np.cumsum(self.kv_len)]), dtype=torch.int32, device=DEV)
        if sum(self.kv_len):
            cp.kv_append(self.kv, torch.cat(self.k).to(DEV), torch.cat(self.v).to(DEV), q_start=starts)

    def positions(self, s):
        return np.arange(self.kv_len[s] - self.new[s], self.kv_len[s])

    def hide(self, window, n_sink):
        """Poisons what no row of a window sees: whole pages are given back (the
        table names none), and single keys become NaN."""
        for s, t in enumerate(self.kv_len):
            first = max(0, t - self.new[s] - window + 1)
            for j in range(min(n_sink, t), first):
                page = int(self.tables[s, j // B])
                if page >= 0:
                    self.kc[page, j % B] = float("nan")
                    self.vc[page, j % B] = float("inf")
            for b in range(-(-n_sink // B), first // B):
                self.tables[s, b] = -1
        self.dev_tables.copy_(self.tables)

    def run(self, window=0, n_sink=0, scale=0.0, lse=True, ws=None):
        q = self.q.to(DEV)
        o = torch.full((len(q), self.Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        s = torch.full((len(q), self.Hq), float("nan"), device=DEV) if lse else None
        if ws is None:
            size = cp.attn_paged_workspace_size(self.kv, len(q), self.max_q, self.Hq)
            ws = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
        cp.attn_paged(self.kv, q, o, ws, lse=s, q_start=self.q_start, max_q=self.max_q, window=window, n_sink=n_sink,
                      softmax_scale=scale)
        return o, s

    def check(self, o, lse, window=0, n_sink=0, scale=None, rows=None):
        """Every row (or `rows` of each sequence) against the oracle, by its bounds."""
        o, lse = f64(o), None if lse is None else f64(lse)
        for s, t in enumerate(self.kv_len):
            idx = np.arange(self.new[s]) if rows is None else np.unique(np.clip(rows, 0, max(0, self.new[s] - 1)))
            if not self.new[s]:
                continue
            r = self.start[s] + idx
            want = owin.attend(f64(self.q)[r], self.positions(s)[idx], f64(self.k[s]), f64(self.v[s]), np.arange(t),
                               window, n_sink, scale)
            compare(o[r], None if lse is None else lse[r], want, t, f"sequence {s} ({t} positions, {self.new[s]} rows)")


def compare(o, lse, want, n_keys, what):
    wo, wl, a, s = want
    on_o, on_lse = owin.bounds(wo, wl, a, s, n_keys)
    empty = np.isneginf(wl)
    assert np.array_equal(np.isnan(o), np.isnan(wo)), f"{what}: NaN"
    assert (o[empty] == 0).all(), f"{what}: rows without keys"
    with np.errstate(invalid="ignore"):
        err = np.abs(o - wo) / on_o
    assert np.nanmax(err, initial=0.0) <= 1.0, f"{what}: O off by {np.nanmax(err):.3g} of its bound"
    if lse is not None:
        assert np.array_equal(np.isneginf(lse), empty), f"{what}: LSE of empty rows"
        err = np.abs(lse[~empty] - wl[~empty]) / on_lse[~empty]
        assert err.max(initial=0.0) <= 1.0, f"{what}: LSE off by {err.max():.3g} of its bound"
