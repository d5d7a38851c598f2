"""The operators over sequences that share pages of one cache, as measured cases.

Five operators: `fork`, `reserve` (copy on write), `release` and `compact` of the page ledger, and `attend`, block attention in
which the pages that a group of sequences has in common are read once for all of them.  A case is one call as a serving
program makes it.  `run` computes it in plain torch operations, or, with `own`, through the framework's entry points.

Layouts: a pool is [layer][page][kv head][K | V][16 * hd] with K as [hd/8][16 keys][8 dims] and V as [hd/16][4][16 dims][4 keys]
(key = 4 * second + fourth index); a block table row lists a sequence's pages, -1 = none; page_refs counts the entries that
hold a page.
"""
import math
import types

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16


# ---- cases --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # single tokens of a handful of samples of one short prompt, small fp32 model: launches
        {"name": "attend_token_f32", "op": "attend", "dtype": "f32", "heads": 4, "kv_heads": 4, "hd": 64, "seqs": 4, "groups": 1, "rows": 1,
         "prefix_lo": 128, "prefix_hi": 128, "own_lo": 1, "own_hi": 27, "causal": True},
        # plain decoding of 32 requests under one 8k system prompt, attention shape of the 8B target: the prefix's bytes
        {"name": "attend_token_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "seqs": 32, "groups": 1, "rows": 1,
         "prefix_lo": 8192, "prefix_hi": 8192, "own_lo": 40, "own_hi": 613, "causal": True},
        # draft blocks (no mask) of 16 requests under two prompts, contexts of 1k to 4k as in the ragged benchmark configuration
        {"name": "attend_draft_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "seqs": 16, "groups": 2, "rows": 16,
         "prefix_lo": 1029, "prefix_hi": 2900, "own_lo": 25, "own_hi": 1190, "causal": False},
        # verification of 32 blocks of 16 under one 16k document: arithmetic
        {"name": "attend_verify_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "seqs": 32, "groups": 1, "rows": 16,
         "prefix_lo": 16384, "prefix_hi": 16384, "own_lo": 100, "own_hi": 1531, "causal": True},
        # one more sample of a short prompt
        {"name": "fork_one", "op": "fork", "dtype": "f32", "layers": 2, "draft_layers": 1, "kv_heads": 4, "hd": 64, "parents": 1, "children": 1,
         "len_lo": 131, "len_hi": 131, "tokens": 8},
        # sixteen samples of each of four documents
        {"name": "fork_wide", "op": "fork", "dtype": "bf16", "layers": 1, "draft_layers": 1, "kv_heads": 1, "hd": 16, "parents": 4, "children": 60,
         "len_lo": 8192, "len_hi": 16384, "tokens": 16},
        # the pages behind three samples of a short prompt, small fp32 model
        {"name": "reserve_f32", "op": "reserve", "dtype": "f32", "layers": 2, "draft_layers": 1, "kv_heads": 4, "hd": 64, "parents": 1, "children": 3,
         "len_lo": 131, "len_hi": 131, "tokens": 8},
        # the first block after 28 samples were forked off four prompts: the whole 36 + 5 layer cache of the 8B models
        {"name": "reserve_8b", "op": "reserve", "dtype": "bf16", "layers": 36, "draft_layers": 5, "kv_heads": 8, "hd": 128, "parents": 4, "children": 28,
         "len_lo": 405, "len_hi": 643, "tokens": 16},
        # a finished request
        {"name": "release_one", "op": "release", "dtype": "f32", "layers": 2, "draft_layers": 1, "kv_heads": 4, "hd": 64, "parents": 2, "children": 1,
         "len_lo": 128, "len_hi": 211, "tokens": 8},
        # sixty samples that lost
        {"name": "release_wide", "op": "release", "dtype": "bf16", "layers": 1, "draft_layers": 1, "kv_heads": 1, "hd": 16, "parents": 4, "children": 60,
         "len_lo": 8192, "len_hi": 16384, "tokens": 16},
        # closing the holes of a small pool
        {"name": "compact_f32", "op": "compact", "dtype": "f32", "layers": 2, "draft_layers": 1, "kv_heads": 4, "hd": 64, "parents": 6, "children": 2,
         "len_lo": 40, "len_hi": 211, "tokens": 8, "pages": 128},
        # ... and of a pool of the 8B models that is half in use
        {"name": "compact_8b", "op": "compact", "dtype": "bf16", "layers": 36, "draft_layers": 5, "kv_heads": 8, "hd": 128, "parents": 8, "children": 8,
         "len_lo": 90, "len_hi": 410, "tokens": 16, "pages": 256},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "fork", "reserve", "release", "compact"])
    if op == "attend":
        bf16 = rng.random() < 0.75
        heads, kv = rng.choice([(32, 8), (32, 4), (16, 2), (8, 8), (12, 4), (4, 4), (24, 3), (10, 2)])
        hd = rng.choice([64, 128, 128, 128, 96, 32, 80]) if bf16 else rng.choice([64, 32, 128, 48])
        rows = min(rng.choice([1, 1, rng.randint(2, 15), rng.randint(2, 15), 16]), 64 // (heads // kv))
        seqs = _log_int(rng, 1, 48)
        groups = rng.randint(1, min(4, seqs))
        hi = _log_int(rng, 16, 16384 if bf16 else 2048)
        c = {"op": op, "dtype": "bf16" if bf16 else "f32", "heads": heads, "kv_heads": kv, "hd": hd, "seqs": seqs, "groups": groups, "rows": rows,
             "prefix_lo": rng.randint(max(1, hi // 3), hi), "prefix_hi": hi, "own_lo": rng.randint(0, 20), "own_hi": _log_int(rng, 24, 1500),
             "causal": rng.random() < 0.6}
        most = work(listed()[3])["flops"] * (1.0 if bf16 else 0.05)
        while work(c)["flops"] > most:
            c["prefix_lo"], c["prefix_hi"], c["own_hi"] = c["prefix_lo"] // 2, c["prefix_hi"] // 2, c["own_hi"] // 2 + 12
        return c
    bf16 = rng.random() < 0.75
    small = rng.random() < 0.5
    parents = _log_int(rng, 1, 8)
    c = {"op": op, "dtype": "bf16" if bf16 else "f32", "layers": rng.randint(1, 4) if small or not bf16 else rng.randint(5, 32),
         "draft_layers": rng.randint(1, 3 if small else 5), "kv_heads": rng.choice([1, 2, 4, 4, 8]), "hd": rng.choice([32, 64, 128, 128, 96, 80]),
         "parents": parents, "children": _log_int(rng, 1, 24 if op in ("reserve", "compact") else 60),
         "len_lo": rng.randint(1, 130), "len_hi": _log_int(rng, 140, 600 if op in ("reserve", "compact") else 16000), "tokens": rng.randint(1, 16)}
    if op in ("fork", "release"):
        c.update(layers=1, draft_layers=1, kv_heads=1, hd=16)
    if op == "compact":
        c["parents"], c["len_hi"] = min(parents + 1, 6), min(c["len_hi"], 420)
        c["pages"] = 2 * _need(c) + rng.randint(1, 40)
    return c


def _spread(n, lo, hi):
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _shape(c):
    """Lengths, groups and shared pages of an attention case."""
    S, G = c["seqs"], c["groups"]
    starts = [S * g * (g + 1) // (G * (G + 1)) for g in range(G)] + [S]          # groups of growing size
    for g in range(1, G):
        starts[g] = max(starts[g], starts[g - 1] + 1)
    prefix = _spread(G, c["prefix_lo"], c["prefix_hi"])
    grp = [max(g for g in range(G) if starts[g] <= s) for s in range(S)]
    shared = [p // PAGE for p in prefix]
    lens = [shared[grp[s]] * PAGE + x for s, x in enumerate(_spread(S, c["own_lo"], c["own_hi"]))]
    return starts, grp, shared, lens


def _lens(c):
    return _spread(c["parents"], c["len_lo"], c["len_hi"])


def _need(c):
    """Pages that a ledger case holds and asks for."""
    tail = (c["tokens"] + 15) // PAGE + 2
    return sum((n + 15) // PAGE for n in _lens(c)) + (c["parents"] + c["children"]) * tail


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _page_bytes(c):
    return (c["layers"] + c["draft_layers"]) * c["kv_heads"] * 2 * PAGE * c["hd"] * _esize(c)


def work(c):
    if c["op"] == "attend":
        starts, grp, shared, lens = _shape(c)
        R, Hq, hd, S = c["rows"], c["heads"], c["hd"], c["seqs"]
        keys = sum(sum(n + (j + 1 if c["causal"] else R) for j in range(R)) for n in lens)
        tokens = sum(x * PAGE for x in shared) + sum(n + R - shared[grp[s]] * PAGE for s, n in enumerate(lens))
        return {"bytes": (2 * S * R * Hq * hd + 2 * tokens * c["kv_heads"] * hd) * _esize(c), "flops": 4 * hd * Hq * keys}
    lens, P, K = _lens(c), c["parents"], c["children"]
    held = [(n + 15) // PAGE for n in lens]
    forked = [held[i % P] for i in range(K)]
    row = 4 * _width(c)
    if c["op"] == "fork":
        return {"bytes": 4 * sum(held) + K * row + 8 * sum(held) + 16 * K, "flops": 0}
    if c["op"] == "release":
        return {"bytes": 4 * sum(forked) * 2 + 8 * sum(held) + 8 * K, "flops": 0}
    if c["op"] == "reserve":
        copies = [(n % PAGE + 3) // 4 * 4 for n in (lens[i % P] for i in range(K)) if n % PAGE]
        return {"bytes": 2 * sum(copies) * _page_bytes(c) // PAGE + 8 * (P + K) + 4 * (sum(held) + 2 * K), "flops": 0}
    live = sum(held) + sum(1 for i in range(K) if lens[i % P] % PAGE)
    moves = live * (c["pages"] - live) // c["pages"]          # expected over random places
    return {"bytes": 2 * moves * _page_bytes(c) + 8 * c["pages"], "flops": 0}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _width(c):
    """Entries of a block table row."""
    return max((n + c["tokens"] + 31) // PAGE for n in _lens(c))


def _dims(c, layers):
    heads = c.get("heads", c["kv_heads"] * (2 if c["hd"] % 32 else 1))
    return types.SimpleNamespace(n_layers=layers, d_model=64, n_q_heads=heads, n_kv_heads=c["kv_heads"], head_dim=c["hd"], d_ffn=64, vocab=64,
                                 rope_theta=1e4, rms_eps=1e-6, qk_norm=False, n_experts=0, top_k=0, d_expert=0)


def _engine(c, block, seqs, width, n_pages, layers, draft_layers, target_pool, draft_pool):
    """The framework's context over given pool contents (the attention and ledger calls need no weights)."""
    import paper_2602_06036_amd as dfl
    e = dfl.Engine(_dims(c, layers), _dims(c, draft_layers), c["dtype"], block, seqs, width, n_pages, (0,), 63, DEV).create()
    for mine, given in ((e.target_pool, target_pool), (e.draft_pool, draft_pool)):
        if given is not None:
            mine.view(given.dtype).copy_(given.reshape(-1))
    return e


def _tdt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _attend_inputs(c, seed):
    starts, grp, shared, lens = _shape(c)
    S, R = c["seqs"], c["rows"]
    block = max(2, R)
    width = max(lens) // PAGE + (block + 15) // PAGE + 1
    held = [(n + R + 15) // PAGE for n in lens]
    n_pages = sum(shared) + sum(h - shared[grp[s]] for s, h in enumerate(held)) + 3
    ids = np.random.RandomState(seed % (1 << 31)).permutation(n_pages).astype(np.int32)
    at, common = 0, []
    for x in shared:
        common.append(ids[at:at + x])
        at += x
    table = np.full((S, width), -1, np.int32)
    for s in range(S):
        k, own_pages = shared[grp[s]], held[s] - shared[grp[s]]
        table[s, :k] = common[grp[s]]
        table[s, k:held[s]] = ids[at:at + own_pages]
        at += own_pages
    g = _gen(seed)
    st = types.SimpleNamespace(lens=lens, block=block, width=width, n_pages=n_pages, starts=starts, shared=shared, grp=grp)
    # rows after norm and rotation: unit keys and values, queries that single some keys out (scores of spread 2)
    st.pool = torch.randn((2, n_pages, c["kv_heads"], 2, PAGE * c["hd"]), generator=g, device=DEV, dtype=torch.float32).to(_tdt(c))
    st.q = (2.0 * torch.randn((S, R, c["heads"], c["hd"]), generator=g, device=DEV, dtype=torch.float32)).to(_tdt(c))
    st.table = torch.from_numpy(table).to(DEV)
    st.seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    return st


def _ledger_inputs(c, seed):
    """Parents with cached prompts; for `release`, `reserve` and `compact` the children are forked off already (child i of parent i % P), for
    `compact` they have a tail of their own."""
    P, K, lens = c["parents"], c["children"], _lens(c)
    width, rows = _width(c), P + K
    n_pages = c.get("pages") or _need(c) + 5
    ids = np.random.RandomState(seed % (1 << 31)).permutation(n_pages).astype(np.int32)
    table, ln, anchor, refs = np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32), np.zeros(rows, np.int32), np.zeros(n_pages, np.int32)
    at = 0
    for s in range(P):
        h = (lens[s] + 15) // PAGE
        table[s, :h] = ids[at:at + h]
        refs[ids[at:at + h]] = 1
        at += h
        ln[s], anchor[s] = lens[s], 17 + s
    for i in range(K if c["op"] != "fork" else 0):
        s, p = P + i, i % P
        h = (lens[p] + 15) // PAGE
        table[s], ln[s], anchor[s] = table[p], ln[p], anchor[p]
        if c["op"] == "compact" and lens[p] % PAGE:
            table[s, h - 1] = ids[at]
            at += 1
        refs[table[s, :h]] += 1
    st = types.SimpleNamespace(rows=rows, width=width, n_pages=n_pages)
    saved = torch.from_numpy(np.concatenate([table.reshape(-1), ln, anchor, refs])).to(DEV)
    st.saved, st.ledger = saved, saved.clone()
    a = rows * width
    st.table, st.seq_lens = st.ledger[:a].view(rows, width), st.ledger[a:a + rows]
    st.anchor, st.refs = st.ledger[a + rows:a + 2 * rows], st.ledger[a + 2 * rows:]
    st.parents, st.children = [i % P for i in range(K)], [P + i for i in range(K)]
    st.parents_dev = torch.tensor(st.parents, device=DEV)
    st.children_dev = torch.tensor(st.children, device=DEV)
    st.tokens = torch.full((rows,), c["tokens"], dtype=torch.int32, device=DEV)
    st.granted = torch.zeros(rows, dtype=torch.int32, device=DEV)
    st.n_live = torch.zeros(1, dtype=torch.int32, device=DEV)
    st.target_pool = st.draft_pool = None
    if c["op"] in ("reserve", "compact"):
        g = _gen(seed)
        shape = (n_pages, c["kv_heads"], 2, PAGE * c["hd"])
        st.target_pool = torch.randn((c["layers"],) + shape, generator=g, device=DEV, dtype=_tdt(c))
        st.draft_pool = torch.randn((c["draft_layers"],) + shape, generator=g, device=DEV, dtype=_tdt(c))
    return st


def prepare(case, seed):
    c = dict(case)
    if c["op"] == "attend":
        st = _attend_inputs(c, seed)
        if own:
            # the causal cases read the target's pool, the others the draft's
            st.e = _engine(c, st.block, c["seqs"], st.width, st.n_pages, 2, 2, st.pool if c["causal"] else None, None if c["causal"] else st.pool)
            st.starts_dev = torch.tensor(st.starts[:-1], dtype=torch.int32, device=DEV)
            st.anchor = torch.zeros(c["seqs"], dtype=torch.int32, device=DEV)
            st.out = torch.empty_like(st.q)
            st.batch = st.e.batch(st.seq_lens, st.table, st.anchor, max(st.lens))
            st.groups = st.e.groups(st.starts_dev, max(st.shared) * PAGE)
            st.pool = None
    else:
        st = _ledger_inputs(c, seed)
        if own:
            st.e = _engine(c, max(2, c["tokens"]), st.rows, st.width, st.n_pages, c["layers"], c["draft_layers"], st.target_pool, st.draft_pool)
            st.view = st.e.ledger(st.table, st.seq_lens, st.anchor, st.refs)
            if st.target_pool is not None:
                st.target_pool = st.e.target_pool.view(_tdt(c)).view(st.target_pool.shape)
                st.draft_pool = st.e.draft_pool.view(_tdt(c)).view(st.draft_pool.shape)
    st.case = c
    torch.cuda.synchronize()
    return st


# ---- the operators ------------------------------------------------------------------------------------------------------
def _bits(pool):
    return pool.view(torch.int16 if pool.dtype == torch.bfloat16 else torch.int32)


def run(st):
    c = st.case
    if c["op"] == "attend":
        return _attend_own(st) if own else _attend_plain(st)
    # the scheduler's ledger as it stands before the call (one upload), so that every pass does the same work
    st.ledger.copy_(st.saved)
    out = (_ledger_own if own else _ledger_plain)(st)
    tables = [st.table, st.seq_lens, st.anchor, st.refs]
    if c["op"] in ("reserve", "compact"):
        return tables + [out, _bits(st.target_pool), _bits(st.draft_pool)]
    return tables


def _attend_own(st):
    from paper_2602_06036_amd import binding
    c = st.case
    pool = binding.DFLASH_POOL_TARGET if c["causal"] else binding.DFLASH_POOL_DRAFT
    binding.dflash_group_attention(st.e, st.batch, st.groups, pool, 1, st.q, st.out, causal=c["causal"])
    return st.out


def _ledger_own(st):
    from paper_2602_06036_amd import binding
    op = st.case["op"]
    if op == "fork":
        binding.dflash_pages_fork(st.e, st.view, st.parents, st.children)
    elif op == "release":
        binding.dflash_pages_release(st.e, st.view, st.children)
    elif op == "reserve":
        binding.dflash_pages_reserve(st.e, st.view, st.tokens, st.granted)
        return st.granted
    else:
        binding.dflash_pages_compact(st.e, st.view, st.n_live)
        return st.n_live


def _attend_plain(st):
    """Sequence by sequence in fp32: scores, mask, exponentials, weighted sum."""
    c = st.case
    S, R, Hq, Hkv, hd = c["seqs"], c["rows"], c["heads"], c["kv_heads"], c["hd"]
    G = Hq // Hkv
    pool = st.pool[1]                                               # layer 1
    out = torch.empty_like(st.q)
    for s in range(S):
        n = st.lens[s] + R
        pages = pool[st.table[s, :(n + PAGE - 1) // PAGE].long()].float()
        k = pages[:, :, 0].view(-1, Hkv, hd // 8, PAGE, 8).permute(1, 0, 3, 2, 4).reshape(Hkv, -1, hd)[:, :n]
        v = pages[:, :, 1].view(-1, Hkv, hd // 16, 4, 16, 4).permute(1, 0, 3, 5, 2, 4).reshape(Hkv, -1, hd)[:, :n]
        q = st.q[s].float().view(R, Hkv, G, hd).transpose(0, 1).reshape(Hkv, R * G, hd)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
        if c["causal"]:
            last = st.lens[s] + torch.arange(R, device=DEV).repeat_interleave(G)
            x = x.masked_fill(torch.arange(n, device=DEV)[None, :] > last[:, None], float("-inf"))
        p = (x - x.amax(-1, keepdim=True)).exp()
        o = torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)
        out[s] = o.view(Hkv, R, G, hd).transpose(0, 1).reshape(R, Hq, hd).to(out.dtype)
    return out


def _held(st, table):
    return (table >= 0) & (table < st.n_pages)


def _count(st, ids, by):
    st.refs.scatter_add_(0, ids.clamp(min=0).long().reshape(-1), by.to(torch.int32).reshape(-1))


def _ledger_plain(st):
    c = st.case
    if c["op"] == "fork":
        old = st.table[st.children_dev]
        _count(st, old, -_held(st, old).int())
        lens = st.seq_lens[st.parents_dev]
        use = torch.arange(st.width, device=DEV)[None, :] < ((lens + 15) // PAGE)[:, None]
        new = torch.where(use, st.table[st.parents_dev], -1)
        _count(st, new, _held(st, new))
        st.table[st.children_dev] = new
        st.seq_lens[st.children_dev] = lens
        st.anchor[st.children_dev] = st.anchor[st.parents_dev]
    elif c["op"] == "release":
        old = st.table[st.children_dev]
        _count(st, old, -_held(st, old).int())
        st.table[st.children_dev] = -1
        st.seq_lens[st.children_dev] = 0
    elif c["op"] == "reserve":
        return _reserve_plain(st)
    else:
        return _compact_plain(st)


def _reserve_plain(st):
    c, rows = st.case, st.rows
    lens = st.seq_lens.long()
    first = lens // PAGE
    entries = torch.arange((c["tokens"] + 14) // PAGE + 1, device=DEV)[None, :] + first[:, None]
    asked = entries < (lens + st.tokens + 15)[:, None] // PAGE
    at = entries.clamp(max=st.width - 1)
    ids = torch.gather(st.table, 1, at)
    held = _held(st, ids) & asked
    flat = torch.where(held, ids, -1 - torch.arange(ids.numel(), device=DEV, dtype=torch.int32).view_as(ids)).reshape(-1)
    row = torch.arange(rows, device=DEV).repeat_interleave(entries.shape[1])
    rank = ((flat[:, None] == flat[None, :]) & (row[None, :] < row[:, None])).sum(1).view_as(ids)
    shared = held & (rank < st.refs[ids.clamp(min=0).long()] - 1)
    want = shared | (asked & ~held)
    free = (st.refs == 0).nonzero()[:, 0].int()
    taken = want.reshape(-1).cumsum(0).view_as(ids)
    fits = (taken[:, -1] <= free.numel())[:, None]
    new = torch.where(want & fits, free[(taken - 1).clamp(0, free.numel() - 1)], ids)
    move = shared & fits
    _count(st, ids, -move.int())
    _count(st, new, want & fits)
    st.table.scatter_(1, at, torch.where(asked, new, torch.gather(st.table, 1, at)))
    st.granted.copy_((~asked | (_held(st, new) & (st.refs[new.clamp(min=0).long()] == 1))).all(1))
    copied = move & (entries == first[:, None]) & (lens % PAGE != 0)[:, None]
    src, dst = ids[copied].long(), new[copied].long()
    upto = ((lens % PAGE + 3) // 4 * 4)[:, None].expand_as(ids)[copied]
    key = torch.arange(PAGE, device=DEV)
    for pool in (st.target_pool, st.draft_pool):
        hd = c["hd"]
        k = pool[:, :, :, 0].view(pool.shape[0], -1, c["kv_heads"], hd // 8, PAGE, 8)
        v = pool[:, :, :, 1].view(pool.shape[0], -1, c["kv_heads"], hd // 16, 4, 16, 4)
        mk = (key[None, :] < upto[:, None]).view(1, -1, 1, 1, PAGE, 1)
        mv = (key[None, ::4] < upto[:, None]).view(1, -1, 1, 1, 4, 1, 1)
        k[:, dst] = torch.where(mk, k[:, src], k[:, dst])
        v[:, dst] = torch.where(mv, v[:, src], v[:, dst])
    return st.granted


def _compact_plain(st):
    live = st.refs > 0
    n = live.sum()
    ids = torch.arange(st.n_pages, device=DEV)
    src, dst = (live & (ids >= n)).nonzero()[:, 0], (~live & (ids < n)).nonzero()[:, 0]
    to = ids.int()
    to[src] = dst.int()
    st.table.copy_(torch.where(_held(st, st.table), to[st.table.clamp(min=0).long()], st.table))
    st.refs[dst] = st.refs[src]
    st.refs[src] = 0
    for pool in (st.target_pool, st.draft_pool):
        pool[:, dst] = pool[:, src]
    st.n_live.copy_(n)
    return st.n_live


# ---- from the definition, in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    return _attend_exact(c, _attend_inputs(c, seed)) if c["op"] == "attend" else _ledger_exact(c, _ledger_inputs(c, seed))


def _attend_exact(c, st):
    R, Hq, Hkv, hd = c["rows"], c["heads"], c["kv_heads"], c["hd"]
    d = torch.arange(hd, device=DEV)
    out = torch.empty(st.q.shape, dtype=torch.float64, device=DEV)
    flat = st.pool[1].reshape(-1)
    for s, n_s in enumerate(st.lens):
        pos = torch.arange(n_s + R, device=DEV)
        key = pos % PAGE
        page = st.table[s].long()[pos // PAGE]
        for h in range(Hkv):
            base = ((page * Hkv + h) * 2 * PAGE * hd)[:, None]
            K = flat[base + d // 8 * 128 + key[:, None] * 8 + d % 8].double()
            V = flat[base + PAGE * hd + d // 16 * 256 + key[:, None] // 4 * 64 + d % 16 * 4 + key[:, None] % 4].double()
            for j in range(R):
                seen = n_s + j + 1 if c["causal"] else n_s + R
                q = st.q[s, j, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)].double()
                w = torch.softmax(q @ K[:seen].T / hd ** 0.5, dim=1)
                out[s, j, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] = w @ V[:seen]
    return out


def _ledger_exact(c, st):
    """Entry by entry on the host."""
    table, lens, anchor, refs = st.table.cpu().numpy().copy(), st.seq_lens.cpu().numpy().copy(), st.anchor.cpu().numpy().copy(), st.refs.cpu().numpy().copy()
    copies, more = [], None

    def give_back(r):
        for p in range(st.width):
            if table[r, p] >= 0:
                refs[table[r, p]] -= 1
            table[r, p] = -1

    if c["op"] == "fork":
        for a, b in zip(st.parents, st.children):
            give_back(b)
            for p in range(-(-int(lens[a]) // PAGE)):
                table[b, p] = table[a, p]
                refs[table[b, p]] += 1
            lens[b], anchor[b] = lens[a], anchor[a]
    elif c["op"] == "release":
        for r in st.children:
            give_back(r)
            lens[r] = 0
    elif c["op"] == "reserve":
        free, before, seen, granted, stuck = [i for i in range(st.n_pages) if refs[i] == 0], refs.copy(), {}, [], False
        ranges = []
        for r in range(st.rows):
            n = int(lens[r])
            want, ranges_r = [], range(n // PAGE, -(-(n + c["tokens"]) // PAGE))
            for p in ranges_r:
                i = int(table[r, p])
                if i < 0 or seen.get(i, 0) < before[i] - 1:
                    want.append(p)
            for p in ranges_r:
                if table[r, p] >= 0:
                    seen[int(table[r, p])] = seen.get(int(table[r, p]), 0) + 1
            stuck = stuck or len(want) > len(free)
            ranges.append(ranges_r)
            for p in want if not stuck else ():
                i, new = int(table[r, p]), free.pop(0)
                if i >= 0:
                    refs[i] -= 1
                    if p == n // PAGE and n % PAGE:
                        copies.append((i, new, -(-(n % PAGE) // 4) * 4))
                table[r, p], refs[new] = new, 1
        granted = [int(all(table[r, p] >= 0 and refs[table[r, p]] == 1 for p in ranges[r])) for r in range(st.rows)]
        more = torch.tensor(granted, dtype=torch.int32, device=DEV)
    else:
        alive = [i for i in range(st.n_pages) if refs[i] > 0]
        n = len(alive)
        holes = [i for i in range(n) if refs[i] <= 0]
        for a, b in zip([i for i in alive if i >= n], holes):
            copies.append((a, b, PAGE))
            table[table == a] = b
            refs[b], refs[a] = refs[a], 0
        more = torch.tensor([n], dtype=torch.int32, device=DEV)
    out = [torch.from_numpy(x).to(DEV) for x in (table, lens, anchor, refs)]
    if c["op"] in ("fork", "release"):
        return out
    key = torch.arange(PAGE * c["hd"], device=DEV)
    key_k, key_v = key // 8 % PAGE, key // 64 % 4 * 4 + key % 4
    for pool in (st.target_pool, st.draft_pool):
        for a, b, upto in copies:
            for part, of in ((0, key_k), (1, key_v)):
                at = (of < upto).nonzero()[:, 0]
                pool[:, b, :, part, at] = pool[:, a, :, part, at]
    return out + [more, _bits(st.target_pool), _bits(st.draft_pool)]
