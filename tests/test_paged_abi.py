"""Refusals of the calls over a paged cache that need no GPU: every case fails
host-side validation, before any HIP call."""

import ctypes

import pytest
import torch

from paper_2609_04774_amd import cpattn as cp

FAKE = 1 << 20
OK, INV, UNS, CAP = cp.CP_OK, cp.CP_ERR_INVALID, cp.CP_ERR_UNSUPPORTED, cp.CP_ERR_CAPACITY


def kv(**x):
    f = dict(k_cache=FAKE, v_cache=2 * FAKE, n_blocks=8, tables=3 * FAKE, table_stride=4, kv_len=4 * FAKE, n_seqs=2,
             n_heads_kv=2)
    f.update(x)
    return cp.CpPagedKv(**f)


def paged(k=None, q=FAKE, q_stride=0, n_rows=2, q_start=FAKE, max_q=2, Hq=8, D=128, scale=0.0, window=0, n_sink=0, o=FAKE,
          lse=FAKE, ws=FAKE, ws_bytes=1 << 30):
    k = kv() if k is None else k
    return cp.lib.cp_attn_paged(ctypes.byref(k), q, q_stride, n_rows, q_start, max_q, Hq, D, scale, window, n_sink, o, lse,
                                ws, ws_bytes, None)


@pytest.mark.parametrize("args,status", [
    (dict(k=kv(n_heads_kv=0)), INV), (dict(k=kv(n_heads_kv=3)), INV), (dict(Hq=0), INV), (dict(Hq=8192), UNS),
    (dict(D=64), UNS), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(window=-1), INV), (dict(scale=3e38), INV),
    (dict(n_sink=-1), INV), (dict(n_rows=-1), INV), (dict(k=kv(n_seqs=-1)), INV), (dict(n_rows=(1 << 30) + 1), UNS),
    (dict(n_rows=1 << 30, Hq=64), UNS), (dict(q_start=None, n_rows=3), INV), (dict(max_q=0), INV),
    (dict(q_stride=512), INV), (dict(q_stride=1028), INV), (dict(q_stride=-1024), INV), (dict(k=kv(n_blocks=-1)), INV),
    (dict(k=kv(table_stride=-1)), INV), (dict(q=None), INV), (dict(o=None), INV), (dict(k=kv(k_cache=None)), INV),
    (dict(k=kv(v_cache=None)), INV), (dict(k=kv(tables=None)), INV), (dict(k=kv(kv_len=None)), INV),
    (dict(q=FAKE + 8), INV), (dict(o=FAKE + 8), INV), (dict(k=kv(k_cache=FAKE + 8)), INV), (dict(lse=FAKE + 2), INV),
    (dict(q_start=FAKE + 2), INV), (dict(k=kv(tables=FAKE + 2)), INV), (dict(k=kv(kv_len=FAKE + 2)), INV),
    (dict(ws=None), INV), (dict(ws=FAKE + 128), INV), (dict(ws_bytes=4096), CAP),
])
def test_paged(args, status):
    assert paged(**args) == status
    assert "cp_attn_paged" in cp.last_error()


def test_nothing_to_do():
    assert paged(n_rows=0, q=None, o=None, ws=None) == OK
    assert paged(k=kv(n_seqs=0, tables=None), ws=None) == OK
    assert cp.lib.cp_attn_paged(None, FAKE, 0, 1, None, 1, 8, 128, 0.0, 0, 0, FAKE, FAKE, FAKE, 1 << 30, None) == INV
    assert cp.lib.cp_attn_paged_workspace_size(2, 0, 1, 8, 2) == 0 and not cp.last_error()


def test_workspace_sizes():
    size = cp.lib.cp_attn_paged_workspace_size
    assert size(2, 2, 0, 8, 2) == 0 and cp.last_error()
    assert size(2, 2, 1, 8, 3) == 0 and cp.last_error()
    assert size(-1, 2, 1, 8, 2) == 0 and cp.last_error()
    one = size(2, 2, 1, 8, 2)
    assert 0 < one <= size(2, 64, 32, 8, 2)
    assert paged(q_start=None, n_rows=2, ws_bytes=one - 1) == CAP and str(one) in cp.last_error()
    assert size(2, 64, 64, 8, 2) <= size(2, 1 << 16, 64, 8, 2)  # rows that may be cut into wide blocks
    plan, _ = cp.shard_plan(0, 100, 2, 0)
    assert cp.attn_window_workspace_size(plan, 8, 2) > 0
    with pytest.raises(cp.CpError):
        cp.attn_window_workspace_size(plan, 8, 3)


def window(plan=None, q=FAKE, k=FAKE, v=FAKE, kc=FAKE, vc=FAKE, n_blocks=8, table=FAKE, table_len=2, Hq=8, Hkv=2, D=128,
           scale=0.0, win=4, n_sink=0, o=FAKE, lse=None, order=0, ws=FAKE, ws_bytes=1 << 30):
    plan = cp.shard_plan(32, 100, 2, 0)[0] if plan is None else plan
    return cp.lib.cp_attn_window(ctypes.byref(plan), q, k, v, kc, vc, n_blocks, table, table_len, Hq, Hkv, D, scale, win,
                                 n_sink, o, lse, order, ws, ws_bytes, None)


@pytest.mark.parametrize("args,status", [
    (dict(plan=cp.shard_plan(33, 100, 2, 0)[0]), INV), (dict(plan=cp.shard_plan(0, (1 << 30) + 1, 2, 0)[0]), UNS),
    (dict(plan=cp.shard_plan(0, 1 << 30, 1, 0)[0], Hq=64, Hkv=8, table_len=0), UNS),
    (dict(order=2), INV), (dict(D=64), UNS), (dict(win=-1), INV), (dict(n_sink=-1), INV), (dict(Hkv=3), INV),
    (dict(scale=float("nan")), INV), (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(o=None), INV),
    (dict(kc=None), INV), (dict(vc=None), INV), (dict(table=None), INV), (dict(table_len=1), INV), (dict(n_blocks=-1), INV),
    (dict(table_len=-1), INV), (dict(q=FAKE + 8), INV), (dict(k=FAKE + 8), INV), (dict(kc=FAKE + 8), INV),
    (dict(table=FAKE + 2), INV), (dict(lse=FAKE + 2), INV), (dict(ws=None), INV), (dict(ws_bytes=4096), CAP),
])
def test_window(args, status):
    assert window(**args) == status
    assert "cp_attn_window" in cp.last_error()


def test_window_plan_is_checked():
    plan, _ = cp.shard_plan(32, 100, 2, 0)
    plan.n_rows += 1
    assert window(plan=plan) == INV
    empty, _ = cp.shard_plan(0, 3, 8, 5)
    assert window(plan=empty, q=None, k=None, v=None, o=None, ws=None) == OK


def append(k=None, rows=FAKE, vrows=FAKE, ks=0, vs=0, n=2, q_start=None, D=128):
    k = kv() if k is None else k
    return cp.lib.cp_kv_append(ctypes.byref(k), rows, vrows, ks, vs, n, q_start, D, None)


@pytest.mark.parametrize("args,status", [
    (dict(k=kv(n_heads_kv=0)), INV), (dict(D=4), INV), (dict(D=12), INV), (dict(n=-1), INV), (dict(n=3), INV),
    (dict(n=(1 << 30) + 2), UNS), (dict(ks=128), INV), (dict(vs=260), INV), (dict(rows=None), INV), (dict(vrows=None), INV),
    (dict(rows=FAKE + 8), INV), (dict(k=kv(tables=None)), INV), (dict(k=kv(kv_len=FAKE + 1)), INV),
    (dict(k=kv(n_blocks=-1)), INV), (dict(q_start=FAKE + 1), INV),
])
def test_append(args, status):
    assert append(**args) == status
    assert "cp_kv_append" in cp.last_error()


def pool(**x):
    f = dict(tables=FAKE, table_stride=4, kv_len=2 * FAKE, refs=3 * FAKE, n_blocks=64, n_seqs=3, reserved=0)
    f.update(x)
    return cp.CpKvPool(**f)


def calls(p, n=1, a=FAKE, b=FAKE, c=FAKE, caches=(FAKE,), page=64, ws=FAKE, ws_bytes=1 << 20, n_caches=None):
    """Every call on a pool, with its list arguments a, b, c."""
    ptrs = (ctypes.c_void_p * max(1, len(caches)))(*caches)
    m = len(caches) if n_caches is None else n_caches
    r = ctypes.byref(p)
    return {"cp_kv_reserve": lambda: cp.lib.cp_kv_reserve(r, a, b, n, c, None),
            "cp_kv_fork": lambda: cp.lib.cp_kv_fork(r, ptrs, m, page, a, b, n, c, None),
            "cp_kv_free": lambda: cp.lib.cp_kv_free(r, a, b, c, n, None),
            "cp_kv_compact": lambda: cp.lib.cp_kv_compact(r, ptrs, m, page, ws, ws_bytes, None)}


@pytest.mark.parametrize("p", [pool(n_seqs=-1), pool(table_stride=-1), pool(n_blocks=-1), pool(reserved=1),
                               pool(tables=None), pool(kv_len=None), pool(refs=None), pool(tables=FAKE + 2),
                               pool(kv_len=FAKE + 2), pool(refs=FAKE + 1)])
def test_bad_pools(p):
    for name, call in calls(p).items():
        assert call() == INV and name in cp.last_error()


def test_bad_lists_and_caches():
    for name, call in calls(pool(n_blocks=1 << 31)).items():
        assert call() == UNS
    lists = ("cp_kv_reserve", "cp_kv_fork", "cp_kv_free")
    for args, status in ((dict(n=-1), INV), (dict(n=4097), UNS), (dict(a=None), INV), (dict(b=None), INV),
                         (dict(c=None), INV), (dict(a=FAKE + 2), INV)):
        for name in lists:
            assert calls(pool(), **args)[name]() == status and name in cp.last_error()
    for args in (dict(caches=(None,)), dict(caches=(FAKE + 8,)), dict(page=0), dict(page=24), dict(n_caches=257),
                 dict(n_caches=-1)):
        for name in ("cp_kv_fork", "cp_kv_compact"):
            assert calls(pool(), **args)[name]() == INV and name in cp.last_error()
    assert calls(pool(), ws=None)["cp_kv_compact"]() == INV
    assert calls(pool(), ws=FAKE + 16)["cp_kv_compact"]() == INV
    assert calls(pool(), ws_bytes=64)["cp_kv_compact"]() == CAP
    assert calls(pool(), n=0, a=None, b=None, c=None)["cp_kv_free"]() == OK
    assert calls(pool(n_blocks=0, refs=None), ws=None)["cp_kv_compact"]() == OK
    assert cp.lib.cp_kv_compact_workspace_size(-1) == 0 and cp.last_error()
    assert cp.lib.cp_kv_reserve(None, FAKE, FAKE, 1, FAKE, None) == INV


def test_copy_pages():
    def copy(caches=(FAKE,), n_caches=None, n_blocks=8, page=64, src=FAKE, dst=FAKE, n=2):
        ptrs = (ctypes.c_void_p * max(1, len(caches)))(*caches)
        return cp.lib.cp_kv_copy_pages(ptrs, len(caches) if n_caches is None else n_caches, n_blocks, page, src, dst, n, None)
    for args in (dict(n_caches=0), dict(n_caches=257), dict(caches=(None,)), dict(caches=(FAKE + 4,)), dict(n_blocks=-1),
                 dict(page=0), dict(page=40), dict(n=-1), dict(src=None), dict(dst=None), dict(src=FAKE + 1)):
        assert copy(**args) == INV and "cp_kv_copy_pages" in cp.last_error()
    assert copy(n=0, src=None, dst=None) == OK and copy(n_blocks=0, caches=(None,)) == OK


def test_struct_layouts():
    assert ctypes.sizeof(cp.CpPagedKv) == 6 * 8 + 8
    assert ctypes.sizeof(cp.CpKvPool) == 5 * 8 + 8


def test_binding_refuses_host_tensors():
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        cp.PagedKV(torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16), t, t[0])
    with pytest.raises(ValueError):
        cp.KVPool(t, t[0], t[0])
    with pytest.raises(ValueError):
        cp.kv_copy_pages([], t[0], t[0])
    with pytest.raises(ValueError):
        cp.kv_copy_pages([torch.zeros(4, 64)], t[0], t[0])
    plan, _ = cp.shard_plan(0, 4, 1, 0)
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        cp.attn_window(plan, x, x, x, x, t, 4)
