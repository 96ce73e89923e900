"""The serving operators around the paged KV cache, each in its plain form and
as the library's call.

* ``paged``    attention of every sequence's newest rows -- a chunk of a
               prompt, or one token each -- over its pages, with or without a
               sliding window and a few first tokens that stay visible;
* ``rank``     the same window for one context-parallel rank's zigzag rows:
               keys of the paged cached prefix, then of the new tokens;
* ``append``   the new tokens' K and V, as they lie in a fused projection's
               output, into their sequences' pages;
* ``copy``, ``fork``, ``free``, ``compact``  pages of the cache copied, shared
               with new sequences, given back, and moved to the pool's front.

Every pass starts from the same page tables, lengths and reference counts: a
pass that changes them first restores them from the ones the scheduler holds.
"""

import math

import numpy as np
import torch

own = False

D = 128
B = 16
DEV = "cuda"


def listed():
    return [
        # One user's next token behind an odd 4K context: latency.
        {"name": "decode_1", "kind": "paged", "n": 1, "lens": 1, "new_lo": 1, "new_hi": 1, "ctx_lo": 4100,
         "ctx_hi": 4100, "Hq": 32, "Hkv": 8, "window": 0, "sink": 0},
        # One decoding step of 64 users of very different context lengths.
        {"name": "decode_64", "kind": "paged", "n": 64, "lens": 2, "new_lo": 1, "new_hi": 1, "ctx_lo": 200,
         "ctx_hi": 32768, "Hq": 32, "Hkv": 8, "window": 0, "sink": 0},
        # A step that mixes chunks of prompts with decoding users.
        {"name": "mixed_16", "kind": "paged", "n": 16, "lens": 3, "new_lo": 1, "new_hi": 1100, "ctx_lo": 1,
         "ctx_hi": 8192, "Hq": 32, "Hkv": 8, "window": 0, "sink": 0},
        # The largest: the last 4K chunk of a long prompt.
        {"name": "chunk_4k_after_28k", "kind": "paged", "n": 1, "lens": 4, "new_lo": 4096, "new_hi": 4096,
         "ctx_lo": 28677, "ctx_hi": 28677, "Hq": 32, "Hkv": 8, "window": 0, "sink": 0},
        # A windowed layer's decoding step: 128 users, pages behind the window given back.
        {"name": "window_decode_128", "kind": "paged", "n": 128, "lens": 5, "new_lo": 1, "new_hi": 1, "ctx_lo": 900,
         "ctx_hi": 16384, "Hq": 64, "Hkv": 8, "window": 4096, "sink": 4},
        # A windowed layer of a 32K prompt at degree 4: one rank's rows.
        {"name": "window_32k_c4", "kind": "rank", "P": 0, "R": 32768, "C": 4, "rank": 0, "Hq": 32, "Hkv": 8,
         "window": 4096, "sink": 4},
        # A turn of a conversation in a small slice of a windowed layer, odd everywhere.
        {"name": "window_turn_3001_c2", "kind": "rank", "P": 6000, "R": 3001, "C": 2, "rank": 1, "Hq": 8, "Hkv": 1,
         "window": 1000, "sink": 5},
        # The K and V of a decoding step of 64 users.
        {"name": "append_64", "kind": "append", "n": 64, "lens": 6, "new_lo": 1, "new_hi": 1, "ctx_lo": 1,
         "ctx_hi": 4096, "Hq": 32, "Hkv": 8},
        # The K and V of a large step of ragged prompts.
        {"name": "append_ragged", "kind": "append", "n": 24, "lens": 7, "new_lo": 30, "new_hi": 4096, "ctx_lo": 1,
         "ctx_hi": 1024, "Hq": 32, "Hkv": 8},
        # Eight prompts, eight continuations of each, four layers.
        {"name": "fork_8_to_64", "kind": "fork", "n": 8, "each": 8, "lens": 8, "ctx_lo": 100, "ctx_hi": 4096,
         "pool": 4096, "caches": 8, "Hkv": 8},
        # The pages that 128 users' windows have passed, given back.
        {"name": "free_128", "kind": "free", "n": 128, "lens": 9, "ctx_lo": 100, "ctx_hi": 16384, "window": 2048,
         "sink": 4, "pool": 65536},
        # A pool of which two fifths are in use, scattered, moved to its front; four layers.
        {"name": "compact_4096", "kind": "compact", "n": 24, "lens": 10, "ctx_lo": 300, "ctx_hi": 3000, "pool": 4096,
         "caches": 8, "Hkv": 8},
    ]


MAX_FLOPS = 2.0e12
MAX_BYTES = 1.6e9


def draw(rng):
    """One more case: lengths spread over their logarithm, odd ones among
    them, every head layout, with and without a window."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["decode", "decode", "chunk", "chunk", "rank", "rank", "append", "copy", "fork", "free",
                           "compact"])
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (8, 2), (8, 1), (28, 4), (16, 16)])
        c = {"kind": "paged" if kind in ("decode", "chunk") else kind, "lens": rng.randrange(1 << 20)}
        windowed = rng.random() < 0.4
        mask = {"window": between(16, 8192) if windowed else 0, "sink": rng.randrange(0, 40) if windowed else 0}
        if kind == "decode":
            new = rng.choice([1, 1, 1, rng.randint(2, 6)])
            c.update(n=between(1, 192), new_lo=new, new_hi=new, ctx_lo=between(1, 8192), ctx_hi=between(8192, 65536),
                     Hq=Hq, Hkv=Hkv, **mask)
        elif kind == "chunk":
            c.update(n=between(1, 24), new_lo=between(1, 64), new_hi=between(65, 2048), ctx_lo=between(1, 1024),
                     ctx_hi=between(1025, 32768), Hq=Hq, Hkv=Hkv, **mask)
        elif kind == "rank":
            C = rng.choice([1, 2, 4, 8])
            del c["lens"]
            c.update(P=B * between(1, 1024) if rng.random() < 0.5 else 0, R=between(33, 24576), C=C,
                     rank=rng.randrange(C), Hq=Hq, Hkv=Hkv, window=between(16, 8192), sink=rng.randrange(0, 40))
        elif kind == "append":
            lo = between(1, 512)
            c.update(n=between(1, 256), new_lo=lo, new_hi=lo if rng.random() < 0.5 else between(513, 4096),
                     ctx_lo=between(1, 64), ctx_hi=between(65, 8192), Hq=Hq, Hkv=Hkv)
        elif kind == "free":
            c.update(n=between(2, 256), ctx_lo=between(1, 512), ctx_hi=between(513, 8192), window=between(16, 4096),
                     sink=rng.randrange(0, 40), pool=between(140000, 200000))
        else:
            c.update(pool=between(1024, 6144), caches=2 * rng.randint(1, 6), Hkv=rng.choice([1, 2, 4, 8]))
            if kind == "copy":
                c.update(pages=between(1, c["pool"] // 2))
            elif kind == "fork":
                c.update(n=rng.randint(1, 8), each=rng.randint(1, 12), ctx_lo=between(1, 100), ctx_hi=between(101, 1500))
            else:
                c.update(n=between(1, 16), ctx_lo=between(1, 256), ctx_hi=between(257, 800))
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _plain_values(c) <= 6e9:
            return c


def _plain_values(case):
    """Scores, or values of K, that the plain form holds at once (padded to the longest sequence)."""
    if case["kind"] == "paged":
        new, ctx = _lengths(case)
        return case["n"] * int((new + ctx).max()) * max(case["Hq"] * int(new.max()), 2 * case["Hkv"] * D)
    if case["kind"] == "rank":
        return case["Hq"] * (case["R"] // case["C"] + 2) * (case["P"] + case["R"])
    return 0


# --- shapes -----------------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens before them) of every sequence."""
    rng = np.random.RandomState(case["lens"])

    def spread(lo, hi):
        x = np.exp(rng.uniform(math.log(lo), math.log(hi + 1), case["n"]))
        return np.clip(x.astype(np.int64), lo, hi)

    new = spread(case["new_lo"], case["new_hi"]) if "new_lo" in case else np.zeros(case["n"], np.int64)
    return new, spread(case["ctx_lo"], case["ctx_hi"])


def _zigzag(case):
    """Positions (from the first new token) of the rank's rows: chunks `rank`
    and 2C-1-rank of the 2C equal chunks of the padded suffix."""
    R, C, r = case["R"], case["C"], case["rank"]
    s = -(-R // (2 * C))
    chunks = [(c * s, min(R, c * s + s)) for c in (r, 2 * C - 1 - r)]
    return np.concatenate([np.arange(lo, hi) for lo, hi in chunks if hi > lo] or [np.arange(0)])


def _visible(q_pos, window, sink):
    """Keys that a row at each position sees, and one past the last key no row
    sees behind the window (the first is `sink`)."""
    n = q_pos + 1
    return n if not window else np.minimum(n, window + np.clip(np.minimum(n - window, sink), 0, None))


def _seen_keys(first, last, window, sink):
    """Keys of one sequence that some row of positions first .. last sees."""
    if not window:
        return last + 1
    lo = max(0, first - window + 1)
    return last + 1 - lo + min(sink, lo)


def work(case):
    kind = case["kind"]
    if kind == "paged":
        new, ctx = _lengths(case)
        rows = int(new.sum())
        pairs = sum(int(_visible(np.arange(c, c + n), case["window"], case["sink"]).sum()) for n, c in zip(new, ctx))
        keys = sum(_seen_keys(int(c), int(c + n - 1), case["window"], case["sink"]) for n, c in zip(new, ctx))
        return {"flops": 4 * D * case["Hq"] * pairs,
                "bytes": 4 * D * case["Hq"] * rows + 4 * case["Hq"] * rows + 4 * D * case["Hkv"] * keys}
    if kind == "rank":
        pos = case["P"] + _zigzag(case)
        pairs = int(_visible(pos, case["window"], case["sink"]).sum())
        seen = np.zeros(case["P"] + case["R"] + 1, np.int64)  # +1 where a row's window begins, -1 behind it
        np.add.at(seen, np.maximum(0, pos - case["window"] + 1), 1)
        np.add.at(seen, pos + 1, -1)
        seen = np.cumsum(seen)[:-1] > 0
        if len(pos):
            seen[:min(case["sink"], int(pos.max()) + 1)] = True
        return {"flops": 4 * D * case["Hq"] * pairs,
                "bytes": (4 * D + 4) * case["Hq"] * len(pos) + 4 * D * case["Hkv"] * int(seen.sum())}
    if kind == "append":
        new, _ = _lengths(case)
        return {"flops": 0, "bytes": 2 * 4 * D * case["Hkv"] * int(new.sum())}
    if kind == "free":
        _, ctx = _lengths(case)
        pages = np.maximum(0, (ctx - case["window"]) // B - -(-case["sink"] // B))
        return {"flops": 0, "bytes": 16 * int(pages.sum()) + 12 * case["n"]}
    page = 2 * B * D * case["Hkv"] * case["caches"]
    if kind == "copy":
        return {"flops": 0, "bytes": 2 * page * case["pages"]}
    _, ctx = _lengths(case)
    if kind == "fork":
        shared = int((ctx // B).sum()) * case["each"]
        return {"flops": 0, "bytes": 2 * page * int((ctx % B > 0).sum()) * case["each"] + 12 * shared + 4 * case["pool"]}
    live = int((-(-ctx // B)).sum())
    # Of pages scattered over the pool, the share that lies behind the first `live` ones moves.
    return {"flops": 0, "bytes": int(2 * page * live * (1 - live / case["pool"])) + 8 * case["pool"] + 8 * live}


# --- inputs -----------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _fill(g, *shape):
    """Cache contents: drawn for the first 64 MB and repeated, scaled page by page."""
    n = math.prod(shape)
    base = torch.randn(min(n, 1 << 25), generator=g, device=DEV).to(torch.bfloat16)
    out = base.repeat(-(-n // base.numel()))[:n].reshape(shape)
    return out * (0.75 + 0.5 * torch.rand(shape[0], *[1] * (len(shape) - 1), generator=g, device=DEV)).to(torch.bfloat16)


def _tables(g, pages, n_blocks, extra_rows=0):
    """Page tables of sequences that hold so many pages, at random places of the pool; -1 behind them."""
    width = max(1, int(pages.max()))
    t = torch.full((len(pages) + extra_rows, width), -1, dtype=torch.int32, device=DEV)
    has = torch.arange(width, device=DEV)[None] < torch.as_tensor(pages, device=DEV)[:, None]
    perm = torch.randperm(n_blocks, generator=g, device=DEV)[:int(pages.sum())]
    t[:len(pages)][has] = perm.to(torch.int32)
    return t


def _starts(new):
    return torch.as_tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)


def _pool(state, tables, kv_len, n_blocks):
    """The scheduler's tables, lengths and reference counts (one buffer, so that a
    pass restores them with one copy), and the ones that a pass changes."""
    refs = torch.zeros(n_blocks, dtype=torch.int32, device=DEV)
    held = tables[tables >= 0].long()
    refs.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    parts = [tables, kv_len, refs]
    state["before"] = torch.cat([p.reshape(-1) for p in parts])
    state["ints"] = state["before"].clone()
    views, at = [], 0
    for p in parts:
        views.append(state["ints"][at:at + p.numel()].view(p.shape))
        at += p.numel()
    state["tables"], state["kv_len"], state["refs"] = views


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case, "own": {}}
    if kind == "paged":
        new, ctx = _lengths(case)
        total = new + ctx
        pages = -(-total // B)
        n_blocks = int(pages.sum() * 1.1) + 2
        Hq, Hkv = case["Hq"], case["Hkv"]
        lean = 0.5 * torch.randn(1, Hkv, 1, D, generator=g, device=DEV)  # a direction that the first tokens' keys share with the queries
        q = torch.randn(int(new.sum()), Hkv, Hq // Hkv, D, generator=g, device=DEV) + lean
        s["q"] = q.reshape(-1, Hq, D).to(torch.bfloat16)
        s["k_cache"], s["v_cache"] = _fill(g, n_blocks, B, Hkv, D), _fill(g, n_blocks, B, Hkv, D)
        tables = _tables(g, pages, n_blocks)
        s["k_cache"][tables[:, 0].long(), :4] += (4 * lean[:, :, 0]).to(torch.bfloat16)
        if case["window"]:  # pages that the window has passed are given back
            j = torch.arange(tables.shape[1], device=DEV)[None] * B
            first = torch.as_tensor(ctx, device=DEV)[:, None] - case["window"] + 1
            tables = torch.where((j >= case["sink"]) & (j + B <= first), torch.full_like(tables, -1), tables)
        s["tables"], s["kv_len"] = tables, torch.as_tensor(total, dtype=torch.int32, device=DEV)
        s["q_start"] = _starts(new) if case["new_lo"] != case["new_hi"] else None
        s["max_q"], s["max_kv"] = int(new.max()), int(total.max())
    elif kind == "rank":
        P, R, Hq, Hkv = case["P"], case["R"], case["Hq"], case["Hkv"]
        rows = _zigzag(case)
        s["rows"] = torch.as_tensor(rows, device=DEV)
        s["q"] = _randn(g, len(rows), Hq, D)
        s["k_new"], s["v_new"] = _randn(g, R, Hkv, D), _randn(g, R, Hkv, D)
        n_blocks = max(1, P // B + 3)
        s["k_cache"], s["v_cache"] = _fill(g, n_blocks, B, Hkv, D), _fill(g, n_blocks, B, Hkv, D)
        s["table"] = torch.randperm(n_blocks, generator=g, device=DEV)[:P // B].to(torch.int32)
        # The ranks of a request share its output; this rank writes its rows.
        s["o"] = torch.zeros(R, Hq, D, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros(R, Hq, device=DEV)
    elif kind == "append":
        new, ctx = _lengths(case)
        pages = -(-(new + ctx) // B)
        n_blocks = int(pages.sum()) + 2
        s["qkv"] = _randn(g, int(new.sum()), case["Hq"] + 2 * case["Hkv"], D)
        s["k_cache"] = torch.zeros(n_blocks, B, case["Hkv"], D, dtype=torch.bfloat16, device=DEV)
        s["v_cache"] = torch.zeros_like(s["k_cache"])
        s["tables"], s["kv_len"] = _tables(g, pages, n_blocks), torch.as_tensor(new + ctx, dtype=torch.int32, device=DEV)
        s["q_start"] = _starts(new) if case["new_lo"] != case["new_hi"] else None
    elif kind == "free":
        _, ctx = _lengths(case)
        pages = -(-ctx // B)
        tables = _tables(g, pages, case["pool"])
        # Every other sequence is a continuation of its neighbour and shares its first pages.
        pairs = len(ctx) // 2
        common = torch.minimum(*(torch.as_tensor(ctx[i:2 * pairs:2] // (2 * B), device=DEV) for i in (0, 1)))
        share = torch.arange(tables.shape[1], device=DEV)[None] < common[:, None]
        tables[1:2 * pairs:2] = torch.where(share, tables[:2 * pairs:2], tables[1:2 * pairs:2])
        kv_len = torch.as_tensor(ctx, dtype=torch.int32, device=DEV)
        _pool(s, tables, kv_len, case["pool"])
        s["seqs"] = torch.randperm(case["n"], generator=g, device=DEV).to(torch.int32)
        s["begin"] = torch.full((case["n"],), case["sink"], dtype=torch.int32, device=DEV)
        s["end"] = (kv_len[s["seqs"].long()] - case["window"]).clamp(min=0).to(torch.int32)
    else:
        s["caches"] = [_fill(g, case["pool"], B, case["Hkv"], D) for _ in range(case["caches"])]
        if kind == "copy":
            perm = torch.randperm(case["pool"], generator=g, device=DEV).to(torch.int32)
            s["src"], s["dst"] = perm[:case["pages"]].contiguous(), perm[case["pages"]:2 * case["pages"]].contiguous()
        else:
            _, ctx = _lengths(case)
            children = case["n"] * case["each"] if kind == "fork" else 0
            kv_len = torch.zeros(case["n"] + children, dtype=torch.int32, device=DEV)
            kv_len[:case["n"]] = torch.as_tensor(ctx, device=DEV)
            _pool(s, _tables(g, -(-ctx // B), case["pool"], children), kv_len, case["pool"])
            if kind == "fork":
                s["parents"] = torch.arange(case["n"], device=DEV, dtype=torch.int32).repeat_interleave(case["each"])
                s["children"] = case["n"] + torch.randperm(children, generator=g, device=DEV).to(torch.int32)
    return s


# --- the plain forms ----------------------------------------------------------------

def _softmax_attend(q, k, v, seen):
    """q [n, Hkv, G*rows, D], k and v [n, Hkv, keys, D], seen [n, 1, G*rows, keys]:
    (sum of v weighted by e^x / sum e^x, ln sum e^x); zeros and -inf for a row that sees no key."""
    x = (q @ k.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(D)).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (top + total.log()).squeeze(-1)


def _seen(q_pos, k_pos, window, sink):
    """Whether a row at q_pos sees the key at k_pos (broadcast)."""
    seen = k_pos <= q_pos
    return seen & ((k_pos > q_pos - window) | (k_pos < sink)) if window else seen


def _gathered(cache, tables):
    """[n, pages, 16, Hkv, D] through the tables as [n, Hkv, tokens, D] in 32 bits; zeros where a table names no page."""
    x = cache[tables.long().clamp(min=0)].float() * (tables >= 0)[:, :, None, None, None]
    return x.flatten(1, 2).transpose(1, 2).contiguous()


def _plain_paged(s):
    c = s["case"]
    n, Hq, Hkv = c["n"], c["Hq"], c["Hkv"]
    G, Q = Hq // Hkv, s["max_q"]
    start = s["q_start"] if s["q_start"] is not None else torch.arange(n + 1, device=DEV) * Q
    new = (start[1:] - start[:-1]).long()
    i = torch.arange(Q, device=DEV)
    row = (start[:-1, None].long() + i).clamp(max=s["q"].shape[0] - 1)
    q_pos = s["kv_len"][:, None].long() - new[:, None] + i
    used = -(-s["max_kv"] // B)
    k, v = _gathered(s["k_cache"], s["tables"][:, :used]), _gathered(s["v_cache"], s["tables"][:, :used])
    q = s["q"][row].float().view(n, Q, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * Q, D)
    k_pos = torch.arange(k.shape[2], device=DEV)
    seen = _seen(q_pos[:, :, None], k_pos, c["window"], c["sink"]) & (i[None, :, None] < new[:, None, None])
    o, lse = _softmax_attend(q, k, v, seen.repeat(1, G, 1)[:, None])
    o = o.view(n, Hkv, G, Q, D).permute(0, 3, 1, 2, 4).reshape(n, Q, Hq, D)
    lse = lse.view(n, Hkv, G, Q).permute(0, 3, 1, 2).reshape(n, Q, Hq)
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), new, output_size=s["q"].shape[0])
    at = torch.arange(s["q"].shape[0], device=DEV) - start[:-1].long()[seq]
    return {"o": o[seq, at].to(torch.bfloat16), "lse": lse[seq, at]}


def _plain_rank(s):
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G, n = Hq // Hkv, s["q"].shape[0]
    k = torch.cat([_gathered(s["k_cache"], s["table"][None])[0], s["k_new"].float().transpose(0, 1)], 1)[None]
    v = torch.cat([_gathered(s["v_cache"], s["table"][None])[0], s["v_new"].float().transpose(0, 1)], 1)[None]
    q = s["q"].float().view(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(1, Hkv, G * n, D)
    seen = _seen(c["P"] + s["rows"][:, None], torch.arange(c["P"] + c["R"], device=DEV), c["window"], c["sink"])
    o, lse = _softmax_attend(q, k, v, seen.repeat(G, 1)[None, None])
    s["o"][s["rows"]] = o.view(Hkv, G, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D).to(torch.bfloat16)
    s["lse"][s["rows"]] = lse.view(Hkv, G, n).permute(2, 0, 1).reshape(n, Hq)
    return {"o": s["o"], "lse": s["lse"]}


def _plain_append(s):
    c = s["case"]
    rows = s["qkv"].shape[0]
    start = s["q_start"].long() if s["q_start"] is not None else torch.arange(c["n"] + 1, device=DEV) * c["new_lo"]
    seq = torch.repeat_interleave(torch.arange(c["n"], device=DEV), start[1:] - start[:-1], output_size=rows)
    pos = s["kv_len"].long()[seq] - start[1:][seq] + torch.arange(rows, device=DEV)
    page = s["tables"][seq, pos // B].long()
    s["k_cache"][page, pos % B] = s["qkv"][:, c["Hq"]:c["Hq"] + c["Hkv"]]
    s["v_cache"][page, pos % B] = s["qkv"][:, c["Hq"] + c["Hkv"]:]
    return {"k": s["k_cache"], "v": s["v_cache"]}


def _plain_copy(s):
    for x in s["caches"]:
        x[s["dst"].long()] = x[s["src"].long()]
    return s["caches"]


def _plain_free(s):
    s["ints"].copy_(s["before"])
    t, seqs = s["tables"], s["seqs"].long()
    j = torch.arange(t.shape[1], device=DEV)[None] * B
    stop = torch.minimum(j + B, s["kv_len"][seqs][:, None])
    mine = t[seqs]
    drop = (j >= s["begin"][:, None]) & (stop <= s["end"][:, None]) & (j < stop) & (mine >= 0)
    s["refs"].index_add_(0, mine.clamp(min=0).reshape(-1).long(), -drop.reshape(-1).to(torch.int32))
    t[seqs] = torch.where(drop, torch.full_like(mine, -1), mine)
    return {"tables": t, "refs": s["refs"], "kv_len": s["kv_len"]}


def _plain_fork(s):
    s["ints"].copy_(s["before"])
    t, refs = s["tables"], s["refs"]
    parents, children = s["parents"].long(), s["children"].long()
    length = s["kv_len"][parents].long()
    whole, part = length // B, length % B > 0
    free = torch.argsort((refs != 0).to(torch.int32), stable=True)  # the lowest free pages first
    fresh = free[(torch.cumsum(part.long(), 0) - 1).clamp(min=0)]
    j = torch.arange(t.shape[1], device=DEV)[None]
    shared = j < whole[:, None]
    theirs = t[parents]
    refs.index_add_(0, theirs.clamp(min=0).reshape(-1).long(), (shared & (theirs >= 0)).reshape(-1).to(torch.int32))
    refs.index_add_(0, fresh, part.to(torch.int32))
    own_page = torch.where(part[:, None] & (j == whole[:, None]), fresh[:, None].to(torch.int32), torch.full_like(theirs, -1))
    t[children] = torch.where(shared, theirs, own_page)
    s["kv_len"][children] = length.to(torch.int32)
    last = theirs.gather(1, (whole - 1 + part.long())[:, None])[:, 0].long()
    fresh = torch.where(part, fresh, last)  # no part of a page: the parent's last one onto itself
    for x in s["caches"]:
        x[fresh] = x[last]
    return {"caches": s["caches"], "tables": t, "refs": refs, "kv_len": s["kv_len"]}


def _plain_compact(s):
    s["ints"].copy_(s["before"])
    t, refs = s["tables"], s["refs"]
    live = refs > 0
    front = torch.arange(refs.numel(), device=DEV) < live.sum()
    src, dst = torch.nonzero(live & ~front)[:, 0], torch.nonzero(~live & front)[:, 0]
    to = torch.arange(refs.numel(), device=DEV, dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    t.copy_(torch.where(t >= 0, to[t.long().clamp(min=0)], t))
    refs[dst] = refs[src]
    refs[src] = 0
    for x in s["caches"]:
        x[dst] = x[src]
    return {"caches": s["caches"], "tables": t, "refs": refs}


# --- the library's calls ------------------------------------------------------------

def _own_paged(s):
    from paper_2609_04774_amd import cpattn as cp
    c, h = s["case"], s["own"]
    if not h:  # what an engine holds for all of its steps
        h["kv"] = cp.PagedKV(s["k_cache"], s["v_cache"], s["tables"], s["kv_len"])
        h["o"], h["lse"] = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device=DEV)
        size = cp.attn_paged_workspace_size(h["kv"], s["q"].shape[0], s["max_q"], c["Hq"])
        h["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
    cp.attn_paged(h["kv"], s["q"], h["o"], h["ws"], lse=h["lse"], q_start=s["q_start"], max_q=s["max_q"],
                  window=c["window"], n_sink=c["sink"])
    return {"o": h["o"], "lse": h["lse"]}


def _own_rank(s):
    from paper_2609_04774_amd import cpattn as cp
    c, h = s["case"], s["own"]
    if not h:
        h["plan"] = cp.shard_plan(c["P"], c["R"], c["C"], c["rank"], with_rows=False)[0]
        size = cp.attn_window_workspace_size(h["plan"], c["Hq"], c["Hkv"])
        h["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
    cp.attn_window(h["plan"], s["q"], s["k_new"], s["v_new"], s["o"], h["ws"], c["window"], n_sink=c["sink"],
                   lse=s["lse"], k_cache=s["k_cache"], v_cache=s["v_cache"], block_table=s["table"],
                   out_order=cp.CP_OUT_SEQUENCE)
    return {"o": s["o"], "lse": s["lse"]}


def _own_append(s):
    from paper_2609_04774_amd import cpattn as cp
    c, h = s["case"], s["own"]
    if not h:
        h["kv"] = cp.PagedKV(s["k_cache"], s["v_cache"], s["tables"], s["kv_len"])
    cp.kv_append(h["kv"], s["qkv"][:, c["Hq"]:c["Hq"] + c["Hkv"]], s["qkv"][:, c["Hq"] + c["Hkv"]:],
                 q_start=s["q_start"])
    return {"k": s["k_cache"], "v": s["v_cache"]}


def _own_pool(s):
    from paper_2609_04774_amd import cpattn as cp
    h = s["own"]
    if not h:
        h["pool"] = cp.KVPool(s["tables"], s["kv_len"], s["refs"], caches=s.get("caches", ()))
        h["missing"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        h["ws"] = torch.empty(max(256, cp.kv_compact_workspace_size(h["pool"])), dtype=torch.uint8, device=DEV)
    s["ints"].copy_(s["before"])
    return cp, h


def _own_copy(s):
    from paper_2609_04774_amd import cpattn as cp
    cp.kv_copy_pages(s["caches"], s["src"], s["dst"])
    return s["caches"]


def _own_free(s):
    cp, h = _own_pool(s)
    cp.kv_free(h["pool"], s["seqs"], s["begin"], s["end"])
    return {"tables": s["tables"], "refs": s["refs"], "kv_len": s["kv_len"]}


def _own_fork(s):
    cp, h = _own_pool(s)
    cp.kv_fork(h["pool"], s["parents"], s["children"], h["missing"])
    return {"caches": s["caches"], "tables": s["tables"], "refs": s["refs"], "kv_len": s["kv_len"]}


def _own_compact(s):
    cp, h = _own_pool(s)
    cp.kv_compact(h["pool"], h["ws"])
    return {"caches": s["caches"], "tables": s["tables"], "refs": s["refs"]}


_PLAIN = {"paged": _plain_paged, "rank": _plain_rank, "append": _plain_append, "copy": _plain_copy,
          "fork": _plain_fork, "free": _plain_free, "compact": _plain_compact}
_OWN = {"paged": _own_paged, "rank": _own_rank, "append": _own_append, "copy": _own_copy, "fork": _own_fork,
        "free": _own_free, "compact": _own_compact}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# --- the definition, in 64 bits -------------------------------------------------------

def _exact_rows(q, pos, k, v, window, sink):
    """One KV head's rows q [rows, G, D] at positions pos over keys k, v [keys, D], a block of rows at a time."""
    o, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for a in range(0, len(pos), 512):
        p = pos[a:a + 512]
        lo, hi = (max(0, int(p.min()) - window + 1) if window else 0), int(p.max()) + 1
        at = torch.arange(lo, hi, device=DEV)
        if window and sink and lo:
            at = torch.cat([torch.arange(min(sink, lo), device=DEV), at])
        x = torch.einsum("rgd,kd->rgk", q[a:a + 512], k[at]) / math.sqrt(D)
        hidden = at[None] > p[:, None]
        if window:
            hidden |= (at[None] <= p[:, None] - window) & (at[None] >= sink)
        x = torch.where(hidden[:, None], torch.full_like(x, -math.inf), x)
        lse[a:a + 512] = torch.logsumexp(x, -1)
        w = torch.where(hidden[:, None], torch.zeros_like(x), torch.exp(x - lse[a:a + 512][..., None]))
        o[a:a + 512] = torch.einsum("rgk,kd->rgd", w, v[at])
    return o, lse


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "paged":
        if work(case)["flops"] > 3e12:
            return None
        new, ctx = _lengths(case)
        Hkv, G = case["Hkv"], case["Hq"] // case["Hkv"]
        o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
        r = 0
        for i, (n, c) in enumerate(zip(new.tolist(), ctx.tolist())):
            pages = s["tables"][i, :-(-(n + c) // B)].long()
            pos = torch.arange(c, c + n, device=DEV)
            for h in range(Hkv):
                k, v = (x[pages.clamp(min=0), :, h].reshape(-1, D)[:n + c].double() for x in (s["k_cache"], s["v_cache"]))
                a, b = _exact_rows(s["q"][r:r + n, h * G:(h + 1) * G].double(), pos, k, v, case["window"], case["sink"])
                o[r:r + n, h * G:(h + 1) * G], lse[r:r + n, h * G:(h + 1) * G] = a, b
            r += n
        return {"o": o, "lse": lse}
    if kind == "rank":
        Hkv, G = case["Hkv"], case["Hq"] // case["Hkv"]
        o, lse = s["o"].double(), s["lse"].double()
        half = len(s["rows"]) if case["C"] == 1 else int((s["rows"] < (case["rank"] + 1) * -(-case["R"] // (2 * case["C"]))).sum())
        pages = s["table"].long()
        for h in range(Hkv):
            k, v = (torch.cat([c[pages, :, h].reshape(-1, D), n[:, h]]).double()
                    for c, n in ((s["k_cache"], s["k_new"]), (s["v_cache"], s["v_new"])))
            for part in (slice(0, half), slice(half, None)):
                rows = s["rows"][part]
                if len(rows):
                    a, b = _exact_rows(s["q"][part, h * G:(h + 1) * G].double(), case["P"] + rows, k, v, case["window"], case["sink"])
                    o[rows, h * G:(h + 1) * G], lse[rows, h * G:(h + 1) * G] = a, b
        return {"o": o, "lse": lse}
    if kind == "append":
        new, ctx = _lengths(case)
        out = {"k": s["k_cache"].double(), "v": s["v_cache"].double()}
        r = 0
        for i, (n, c) in enumerate(zip(new.tolist(), ctx.tolist())):
            at = torch.arange(c, c + n, device=DEV)
            slot = s["tables"][i].long()[at // B] * B + at % B
            out["k"].flatten(0, 1)[slot] = s["qkv"][r:r + n, case["Hq"]:case["Hq"] + case["Hkv"]].double()
            out["v"].flatten(0, 1)[slot] = s["qkv"][r:r + n, case["Hq"] + case["Hkv"]:].double()
            r += n
        return out
    if kind == "free":
        return None
    # Pages are copied whole: which go where, one after the other on the host.
    moves = []
    if kind == "copy":
        moves = list(zip(s["src"].tolist(), s["dst"].tolist()))
    else:
        tables, kv_len, refs = s["tables"].tolist(), s["kv_len"].tolist(), s["refs"].tolist()
        free = [p for p, r in enumerate(refs) if r == 0]
        if kind == "fork":
            for p in s["parents"].tolist():
                if kv_len[p] % B:
                    moves.append((tables[p][kv_len[p] // B], free.pop(0)))
        else:
            live = sum(r > 0 for r in refs)
            behind = [p for p, r in enumerate(refs) if r > 0 and p >= live]
            moves = list(zip(behind, free[:len(behind)]))
    src, dst = (torch.as_tensor([m[i] for m in moves], dtype=torch.int64, device=DEV) for i in (0, 1))
    caches = []
    for x in s["caches"]:
        y = x.double()
        y[dst] = x[src].double()
        caches.append(y)
    return caches if kind == "copy" else {"caches": caches, "tables": None, "refs": None, "kv_len": None} if kind == "fork" else {"caches": caches, "tables": None, "refs": None}
