"""The operators over K/V caches that are held in 4 or 8 bits, as measured cases.

Five operators: `attend`, block attention over such a cache; `store`, rows quantised as they are written (and read back); `read`, rows
read back; `park`, the context's own cache of some sequences quantised in all layers and restored to other pages; `restore`, the way back alone.
A case is one call (`store` and `park`: two) as a serving program makes it.  `run` computes it in plain torch operations, or, with `own`,
through the framework's entry points.

What a cache holds: every 32 dims of a row of K or V are a block with a scale 2^(e - 127), one byte e, and 32 codes, of 4 bits (sign, two of exponent, one of
mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) or 8 bits (sign, four of exponent, three of mantissa, up to 448).  e is the least, from 0 on, at which the block's largest
magnitude over its scale is at most 7 (464): half a step above the largest code, so that no element is off by more than half a step there.  Codes round to
nearest, ties to even.  A block with an infinity or a NaN has e = 255 and is NaN.

Layout: [layer][page][kv head][K codes | V codes | K scales | V scales] in bytes, 16 tokens a page, head dims rounded up to NB blocks.  With b = block, d = dim
in the block, key = 4 q + k:
    K, 4 bits:  [b][key][d / 2], the even dim low                     K, 8 bits:  [d / 16][b][key][d % 16]
    V, 4 bits:  [q][d % 16][b][k], the dim below 16 low               V, 8 bits, per pair of blocks: [q][d % 16][b % 2][k][d / 16]
    scales:     [key][NB, of three 4]
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
        # single tokens of two short requests of a small fp32 model: launches
        {"name": "attend_token_f32", "op": "attend", "dtype": "f32", "heads": 4, "kv_heads": 4, "hd": 64, "k_bits": 8, "v_bits": 8, "seqs": 2, "rows": 1,
         "rows_lo": 1, "len_lo": 1, "len_hi": 211, "causal": True},
        # plain decoding of 32 requests of 1k to 32k tokens, attention shape of the 8B target, all in 4 bits: the cache's bytes
        {"name": "attend_token_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 32, "rows": 1,
         "rows_lo": 1, "len_lo": 1000, "len_hi": 32768, "causal": True},
        # verification of draft blocks of 16 requests of up to 4k tokens
        {"name": "attend_block_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 16, "rows": 16,
         "rows_lo": 16, "len_lo": 512, "len_hi": 4096, "causal": True},
        # pieces of two long prompts behind what is cached of them, K in 8 bits and V in 4
        {"name": "attend_prompt_8b", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "hd": 128, "k_bits": 8, "v_bits": 4, "seqs": 2, "rows": 512,
         "rows_lo": 391, "len_lo": 1500, "len_hi": 6007, "causal": True},
        # the new rows of a decoding step of eight requests
        {"name": "store_token_8b", "op": "store", "dtype": "bf16", "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 8, "rows": 1, "rows_lo": 1,
         "len_lo": 5, "len_hi": 3001},
        # one layer's rows of four prompts
        {"name": "store_prompt_8b", "op": "store", "dtype": "bf16", "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 4, "rows": 8192,
         "rows_lo": 1777, "len_lo": 0, "len_hi": 37},
        # a short cache of a small fp32 model
        {"name": "read_f32", "op": "read", "dtype": "f32", "kv_heads": 4, "hd": 64, "k_bits": 8, "v_bits": 4, "seqs": 2, "rows": 120, "rows_lo": 50,
         "len_lo": 52, "len_hi": 130},
        # one layer of eight long caches, as a kernel over plain rows needs them
        {"name": "read_8b", "op": "read", "dtype": "bf16", "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 8, "rows": 16384, "rows_lo": 3000,
         "len_lo": 3001, "len_hi": 16390},
        # a short request of a small fp32 model, put aside and taken up again
        {"name": "park_f32", "op": "park", "dtype": "f32", "layers": 2, "kv_heads": 4, "hd": 64, "k_bits": 8, "v_bits": 8, "seqs": 1, "len_lo": 133,
         "len_hi": 133},
        # two requests of the 8B target, put aside and taken up again
        {"name": "park_8b", "op": "park", "dtype": "bf16", "layers": 36, "kv_heads": 8, "hd": 128, "k_bits": 4, "v_bits": 4, "seqs": 2, "len_lo": 900,
         "len_hi": 2050},
        # the draft's cache of one request taken up again
        {"name": "restore_draft", "op": "restore", "dtype": "bf16", "layers": 5, "kv_heads": 8, "hd": 128, "k_bits": 8, "v_bits": 8, "seqs": 1, "len_lo": 405,
         "len_hi": 405},
        # four requests of the 8B target taken up again
        {"name": "restore_8b", "op": "restore", "dtype": "bf16", "layers": 36, "kv_heads": 8, "hd": 128, "k_bits": 8, "v_bits": 4, "seqs": 4, "len_lo": 700,
         "len_hi": 2050},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "store", "read", "park", "restore"])
    bf16 = rng.random() < 0.75
    k_bits, v_bits = rng.choice([(4, 4), (4, 4), (8, 8), (8, 4)])
    c = {"op": op, "dtype": "bf16" if bf16 else "f32", "hd": rng.choice([64, 128, 128, 128, 96, 32, 80]), "k_bits": k_bits, "v_bits": v_bits}
    if op == "attend":
        c["heads"], c["kv_heads"] = rng.choice([(32, 8), (32, 8), (32, 4), (16, 2), (8, 8), (12, 4), (4, 4), (24, 3), (10, 2)])
        kind = rng.choice(["token", "token", "block", "prompt"])
        c["seqs"] = _log_int(rng, 1, 6 if kind == "prompt" else 48)
        c["rows"] = {"token": 1, "block": rng.randint(2, 16), "prompt": _log_int(rng, 17, 700)}[kind]
        c["rows_lo"] = c["rows"] if kind != "prompt" else rng.randint(1, c["rows"])
        c["len_hi"] = _log_int(rng, 16, {"token": 40000, "block": 12000, "prompt": 8000}[kind] if bf16 else 4000)
        c["len_lo"] = rng.randint(0, c["len_hi"])
        c["causal"] = rng.random() < 0.7
        most_b, most_f = work(listed()[1])["bytes"], work(listed()[3])["flops"] * (1.0 if bf16 else 0.25)
        while work(c)["bytes"] > most_b or work(c)["flops"] > most_f:
            c["len_lo"], c["len_hi"], c["rows"] = c["len_lo"] // 2, c["len_hi"] // 2 + 8, max(1, c["rows"] * 3 // 4)
            c["rows_lo"] = min(c["rows_lo"], c["rows"])
        return c
    c["kv_heads"] = rng.choice([1, 2, 4, 4, 8, 8, 3])
    if op in ("store", "read"):
        c["seqs"] = _log_int(rng, 1, 48)
        c["rows"] = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 9000)])
        c["rows_lo"] = rng.randint(0 if c["rows"] > 1 else 1, c["rows"])
        c["len_lo"], c["len_hi"] = rng.randint(0, 100), _log_int(rng, 101, 4000)
        if op == "read":
            c["len_lo"], c["len_hi"] = c["rows_lo"] + c["len_lo"] + 1, c["rows"] + c["len_hi"]
        while c["seqs"] * c["rows"] > 40000:
            c["seqs"] = max(1, c["seqs"] // 2)
        return c
    c["layers"] = rng.randint(1, 4) if not bf16 or rng.random() < 0.4 else rng.randint(5, 36)
    c["seqs"] = _log_int(rng, 1, 12)
    c["len_hi"] = _log_int(rng, 1, 2000)
    c["len_lo"] = rng.randint(0, c["len_hi"])
    while c["seqs"] > 1 and c["seqs"] * c["len_hi"] > 4000:
        c["seqs"] -= 1
    return c


def _spread(n, lo, hi):
    return [lo + (hi - lo) * i // (n - 1) for i in range(n)] if n > 1 else [hi]


def _lens(c):
    return _spread(c["seqs"], c["len_lo"], c["len_hi"])


def _counts(c):
    """Rows of each sequence: fewest behind the longest cache, but for rows that are read."""
    n = _spread(c["seqs"], c["rows_lo"], c["rows"])
    return n if c["op"] == "read" else n[::-1]


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _blocks(c):
    return (c["hd"] + 31) // 32


def _held(c):
    """Bytes of one token of one kv head, scales of the blocks included."""
    return _blocks(c) * (32 * (c["k_bits"] + c["v_bits"]) // 8 + 2)


def work(c):
    lens, es, hd = _lens(c), _esize(c), c["hd"]
    if c["op"] == "attend":
        counts, Hq = _counts(c), c["heads"]
        keys = sum(k * n + (k * (k + 1) // 2 if c["causal"] else k * k) for n, k in zip(lens, counts))
        tokens = sum(n + k for n, k in zip(lens, counts))
        return {"bytes": 2 * sum(counts) * Hq * hd * es + tokens * c["kv_heads"] * _held(c), "flops": 4 * hd * Hq * keys}
    if c["op"] in ("store", "read"):
        tokens = sum(_counts(c)) * c["kv_heads"]
        return {"bytes": tokens * (2 * hd * es + _held(c)) * (2 if c["op"] == "store" else 1), "flops": 0}
    tokens = sum(lens) * c["kv_heads"] * c["layers"]
    return {"bytes": tokens * (2 * hd * es + _held(c)) * (2 if c["op"] == "park" else 1), "flops": 0}


# ---- the format in plain operations -------------------------------------------------------------------------------------
_FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exp2_of(e):
    """2^(e - 127) of whole numbers e in [0, 254], exactly; 255: NaN."""
    s = torch.where(e > 0, e << 23, 0x400000).to(torch.int32).view(torch.float32)
    return torch.where(e == 255, float("nan"), s)


def _quantise(x, bits):
    """[..., hd] -> codes [..., NB, 32], scale bytes [..., NB]."""
    x = x.float()
    nb = (x.shape[-1] + 31) // 32
    if x.shape[-1] % 32:
        x = torch.cat([x, torch.zeros(x.shape[:-1] + (32 * nb - x.shape[-1],), device=x.device)], -1)
    x = x.reshape(x.shape[:-1] + (nb, 32))
    m = x.abs().amax(-1).view(torch.int32)
    top, above = (2, 0x600000) if bits == 4 else (8, 0x680000)
    e = ((m >> 23) - top + ((m & 0x7FFFFF) > above).int()).clamp(0, 254)
    y = x * ((254 - e) << 23).view(torch.float32).unsqueeze(-1)
    bad = (m >> 23) == 255
    y = torch.where(bad.unsqueeze(-1), 0.0, y)
    a = y.abs()
    if bits == 4:
        code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
        code |= (y < 0).to(torch.uint8) << 3
    else:
        code = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return code, torch.where(bad, 255, e).to(torch.uint8)


def _values(code, e, bits):
    """codes [..., NB, 32], scale bytes [..., NB] -> fp32 values [..., NB * 32]."""
    if bits == 4:
        table = torch.tensor(_FP4 + tuple(-v for v in _FP4), device=code.device)
        x = table[code.long()]
    else:
        x = code.view(torch.float8_e4m3fn).float()
    return (x * _exp2_of(e.int()).unsqueeze(-1)).flatten(-2)


def _lay_k(code, bits):
    """[..., 16 keys, NB, 32] -> bytes [..., n]."""
    lead, nb = code.shape[:-3], code.shape[-2]
    if bits == 4:
        c = code.reshape(lead + (16, nb, 16, 2))
        return (c[..., 0] | c[..., 1] << 4).transpose(-2, -3).flatten(-3)
    return code.reshape(lead + (16, nb, 2, 16)).movedim(-2, -4).transpose(-2, -3).flatten(-4)


def _lay_v(code, bits):
    lead, nb = code.shape[:-3], code.shape[-2]
    c = code.reshape(lead + (4, 4, nb, 2, 16))                       # q, k, b, half, n
    if bits == 4:
        return (c[..., 0, :] | c[..., 1, :] << 4).movedim(-1, -3).transpose(-1, -2).flatten(-4)          # q, n, b, k
    c = c.movedim(-1, -4)                                             # q, n, k, b, half
    return torch.cat([c[..., b:b + 2, :].transpose(-2, -3).flatten(-5) for b in range(0, nb, 2)], -1)


def _unlay_k(data, nb, bits):
    lead = data.shape[:-1]
    if bits == 4:
        c = data.reshape(lead + (nb, 16, 16)).transpose(-2, -3)      # key, b, byte
        return torch.stack([c & 15, c >> 4], -1).flatten(-2)
    c = data.reshape(lead + (2, nb, 16, 16)).transpose(-2, -3).movedim(-4, -2)      # key, b, half, dim
    return c.flatten(-2)


def _unlay_v(data, nb, bits):
    lead = data.shape[:-1]
    if bits == 4:
        c = data.reshape(lead + (4, 16, nb, 4)).transpose(-1, -2).movedim(-3, -1)      # q, k, b, n
        return torch.stack([c & 15, c >> 4], -2).reshape(lead + (16, nb, 32))
    parts = [data[..., 512 * b:512 * min(b + 2, nb)].reshape(lead + (4, 16, min(2, nb - b), 4, 2)).transpose(-2, -3) for b in range(0, nb, 2)]
    c = torch.cat(parts, -2).movedim(-4, -1)                          # q, k, b, half, n
    return c.reshape(lead + (16, nb, 32))


def _lay_scales(e):
    """[..., 16, NB] -> bytes."""
    if e.shape[-1] == 3:
        e = torch.cat([e, torch.zeros_like(e[..., :1])], -1)
    return e.flatten(-2)


def _places(c):
    """Where K codes, V codes, K scales and V scales begin in a page of a head, and its bytes."""
    nb = _blocks(c)
    k, v, s = 64 * nb * c["k_bits"], 64 * nb * c["v_bits"], 16 * (4 if nb == 3 else nb)
    return 0, k, k + v, k + v + s, k + v + 2 * s


def _pages_of(c, k, v):
    """K and V [..., 16, hd] of pages -> bytes [..., unit]."""
    kc, ke = _quantise(k, c["k_bits"])
    vc, ve = _quantise(v, c["v_bits"])
    return torch.cat([_lay_k(kc, c["k_bits"]), _lay_v(vc, c["v_bits"]), _lay_scales(ke), _lay_scales(ve)], -1)


def _rows_of(c, units):
    """bytes [..., unit] -> K and V in fp32, [..., 16, hd]."""
    nb, hd = _blocks(c), c["hd"]
    p = _places(c)
    e = [units[..., a:b].reshape(units.shape[:-1] + (16, -1))[..., :nb] for a, b in ((p[2], p[3]), (p[3], p[4]))]
    k = _values(_unlay_k(units[..., :p[1]], nb, c["k_bits"]), e[0], c["k_bits"])
    v = _values(_unlay_v(units[..., p[1]:p[2]], nb, c["v_bits"]), e[1], c["v_bits"])
    return k[..., :hd], v[..., :hd]


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _dims(c, layers):
    heads = c.get("heads", c["kv_heads"] * (2 if c["hd"] % 32 else 1))
    return types.SimpleNamespace(n_layers=layers, d_model=64, n_q_heads=heads, n_kv_heads=c["kv_heads"], head_dim=c["hd"], d_ffn=64, vocab=64,
                                 rope_theta=1e4, rms_eps=1e-6, qk_norm=False, n_experts=0, top_k=0, d_expert=0)


def _engine(c, width, n_pages):
    """The framework's context (these calls need no weights)."""
    import paper_2602_06036_amd as dfl
    target, draft = _dims(c, c.get("layers", 1)), _dims(c, 1)
    block = max(2, min(16, 64 // (target.n_q_heads // c["kv_heads"])))
    return dfl.Engine(target, draft, c["dtype"], block, c["seqs"], width, n_pages, (0,), 63, DEV).create()


def _tdt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _rows(c, shape, g):
    """Rows of K or V as a model makes them: some dims of every head larger than the others."""
    loud = 1.0 + 3.0 * (torch.rand((c["kv_heads"], 1, c["hd"]) if shape[-2] == PAGE else (c["kv_heads"], c["hd"]), generator=g, device=DEV) > 0.94)
    return (_randn(shape, g) * loud).to(_tdt(c))


def _table(rng, held, width, n_pages):
    """Block table over pages in random order."""
    ids = rng.permutation(n_pages).astype(np.int32)
    table, at = np.full((len(held), width), -1, np.int32), 0
    for s, h in enumerate(held):
        table[s, :h] = ids[at:at + h]
        at += h
    return torch.from_numpy(table).to(DEV)


def _random_cache(c, layers, n_pages, g):
    """A cache whose pages hold rows of random models, quantised."""
    unit = _places(c)[4]
    data = torch.empty((layers, n_pages, c["kv_heads"], unit), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (c["kv_heads"] * PAGE * c["hd"]))
    for layer in range(layers):
        for p in range(0, n_pages, step):
            shape = (min(step, n_pages - p), c["kv_heads"], PAGE, c["hd"])
            data[layer, p:p + step] = _pages_of(c, _rows(c, shape, g), _rows(c, shape, g))
    return data


def _inputs(c, seed):
    """What both forms and `exact` start from."""
    op, lens, g = c["op"], _lens(c), _gen(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    counts = _counts(c) if op in ("attend", "store", "read") else [0] * c["seqs"]
    st = types.SimpleNamespace(lens=lens, counts=counts)
    held = [(n + (k if op != "read" else 0) + PAGE - 1) // PAGE for n, k in zip(lens, counts)]
    st.n_pages = sum(held) + 3
    st.width = max(held) + 2
    st.table = _table(rng, held, st.width, st.n_pages)
    st.seq_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st.counts_dev = torch.tensor(counts, dtype=torch.int32, device=DEV)
    S, R, H, hd = c["seqs"], c.get("rows", 0), c["kv_heads"], c["hd"]
    if op in ("attend", "read", "restore"):
        st.cache = _random_cache(c, c.get("layers", 1), st.n_pages, g)
    else:
        st.cache = torch.zeros((c.get("layers", 1), st.n_pages, H, _places(c)[4]), dtype=torch.uint8, device=DEV)
    if op == "attend":
        # queries that single some keys out (scores of spread 2)
        st.q = (2.0 * _randn((S, R, c["heads"], hd), g)).to(_tdt(c))
        st.out = torch.zeros_like(st.q)
    if op == "store":
        st.k, st.v = _rows(c, (S, R, H, hd), g), _rows(c, (S, R, H, hd), g)
    if op in ("store", "read"):
        st.k_out, st.v_out = (torch.zeros((S, R, H, hd), dtype=_tdt(c), device=DEV) for _ in range(2))
        # what is read back: the rows just written, or those that end the sequence
        st.starts = torch.tensor(lens if op == "store" else [n - k for n, k in zip(lens, counts)], dtype=torch.int32, device=DEV)
        # the pages that the rows stand in, the rows' places in those, and the rows among all of the call
        first = st.starts.tolist()
        last = [a + k for a, k in zip(first, counts)]
        st.pages = torch.cat([st.table[s, a // PAGE:(b + PAGE - 1) // PAGE] if b > a else st.table[s, :0] for s, (a, b) in enumerate(zip(first, last))]).long()
        behind = np.cumsum([0] + [(b + PAGE - 1) // PAGE - a // PAGE if b > a else 0 for a, b in zip(first, last)]) * PAGE
        st.places_at = torch.from_numpy(np.concatenate([behind[s] + a % PAGE + np.arange(b - a) for s, (a, b) in enumerate(zip(first, last))])).to(DEV)
        st.rows_at = torch.from_numpy(np.concatenate([s * R + np.arange(k) for s, k in enumerate(counts)])).to(DEV)
    if op in ("park", "restore"):
        # the context's pool: the sequences' pages, and those that they come back to
        st.pool_pages = 2 * sum(held) + 3 if op == "park" else st.n_pages
        both = _table(rng, held + held if op == "park" else held, st.width, st.pool_pages)
        st.from_table, st.to_table = both[:S], both[-S:]
        st.from_pages, st.pages, st.to_pages = (torch.cat([t[s, :h] for s, h in enumerate(held)]).long() for t in (st.from_table, st.table, st.to_table))
        st.there = torch.cat([torch.arange(h * PAGE, device=DEV) < n for h, n in zip(held, lens)]).view(-1, 1, PAGE, 1)
        shape = (c["layers"], st.pool_pages, H, 2, PAGE * hd)
        st.pool = torch.zeros(shape, dtype=_tdt(c), device=DEV)
        if op == "park":
            loud = 1.0 + 3.0 * (torch.rand((H, 2, PAGE * hd), generator=g, device=DEV) > 0.94)
            for layer in range(c["layers"]):
                st.pool[layer] = _randn(shape[1:], g) * loud
    return st


def prepare(case, seed):
    c = dict(case)
    st = _inputs(c, seed)
    if own:
        st.e = _engine(c, st.width, getattr(st, "pool_pages", 1))
        anchor = torch.zeros(c["seqs"], dtype=torch.int32, device=DEV)
        longest = max(st.lens)
        st.batch = st.e.batch(st.seq_lens, st.table if c["op"] not in ("park", "restore") else st.from_table, anchor, longest)
        st.kvq = st.e.kvq(st.cache, 0, st.n_pages, c["k_bits"], c["v_bits"])
        if c["op"] in ("park", "restore"):
            mine = st.e.target_pool.view(_tdt(c)).view(st.pool.shape)
            mine.copy_(st.pool)
            st.pool = mine
            st.batch_to = st.e.batch(st.seq_lens, st.to_table, anchor, longest)
        st.keep = anchor
    st.case = c
    torch.cuda.synchronize()
    return st


# ---- the operators ------------------------------------------------------------------------------------------------------
def run(st):
    c = st.case
    (_own if own else _plain)(st)
    if c["op"] == "attend":
        return st.out
    return [st.k_out, st.v_out] if c["op"] in ("store", "read") else st.pool


def _own(st):
    from paper_2602_06036_amd import binding as B
    c = st.case
    if c["op"] == "attend":
        B.dflash_kvq_attention(st.e, st.batch, st.kvq, 0, st.q, st.out, counts=st.counts_dev, causal=c["causal"])
    elif c["op"] == "store":
        B.dflash_kvq_write(st.e, st.batch, st.kvq, 0, st.k, st.v, counts=st.counts_dev)
        B.dflash_kvq_read(st.e, st.batch, st.kvq, 0, st.k_out, st.v_out, starts=st.starts, counts=st.counts_dev)
    elif c["op"] == "read":
        B.dflash_kvq_read(st.e, st.batch, st.kvq, 0, st.k_out, st.v_out, starts=st.starts, counts=st.counts_dev)
    else:
        if c["op"] == "park":
            B.dflash_kvq_pack(st.e, st.batch, st.kvq, st.table)
        B.dflash_kvq_unpack(st.e, st.batch_to, st.kvq, st.table)


def _plain(st):
    {"attend": _attend_plain, "store": _store_plain, "read": _read_plain, "park": _park_plain, "restore": _restore_plain}[st.case["op"]](st)


def _attend_plain(st):
    """Sequence by sequence in fp32: the cache's values, scores, mask, exponentials, weighted sum."""
    c = st.case
    Hq, Hkv, hd = c["heads"], c["kv_heads"], c["hd"]
    G = Hq // Hkv
    st.out.zero_()
    for s in range(c["seqs"]):
        n_s, R = st.lens[s], st.counts[s]
        n = n_s + R
        k, v = _rows_of(c, st.cache[0][st.table[s, :(n + PAGE - 1) // PAGE].long()])          # [pages, heads, 16, hd]
        k = k.transpose(0, 1).reshape(Hkv, -1, hd)[:, :n]
        v = v.transpose(0, 1).reshape(Hkv, -1, hd)[:, :n]
        q = st.q[s, :R].float().view(R, Hkv, G, hd).transpose(0, 1).reshape(Hkv, R * G, hd)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
        if c["causal"]:
            last = n_s + torch.arange(R, device=DEV).repeat_interleave(G)
            x = x.masked_fill(torch.arange(n, device=DEV)[None, :] > last[:, None], float("-inf"))
        p = (x - x.amax(-1, keepdim=True)).exp()
        o = torch.matmul(p, v.contiguous()) / p.sum(-1, keepdim=True)
        st.out[s, :R] = o.view(Hkv, R, G, hd).transpose(0, 1).reshape(R, Hq, hd).to(st.out.dtype)


def _store_plain(st):
    """The pages that the rows stand in, as codes and scales; the new rows put into them; the pages laid out again."""
    c = st.case
    nb, p = _blocks(c), _places(c)
    units = st.cache[0][st.pages]                                        # [pages, heads, unit]
    new = []
    for x, bits, unlay, lay, at, to, sc in ((st.k, c["k_bits"], _unlay_k, _lay_k, 0, p[1], p[2]), (st.v, c["v_bits"], _unlay_v, _lay_v, p[1], p[2], p[3])):
        code, e = _quantise(x.flatten(0, 1)[st.rows_at], bits)           # [rows, heads, NB, 32]
        codes = unlay(units[..., at:to], nb, bits).transpose(1, 2).flatten(0, 1).clone()
        scales = units[..., sc:sc + p[4] - p[3]].unflatten(-1, (PAGE, -1))[..., :nb].transpose(1, 2).flatten(0, 1).clone()
        codes[st.places_at], scales[st.places_at] = code, e
        new.append(lay(codes.unflatten(0, (-1, PAGE)).transpose(1, 2), bits))
        new.append(_lay_scales(scales.unflatten(0, (-1, PAGE)).transpose(1, 2)))
    st.cache[0][st.pages] = torch.cat([new[0], new[2], new[1], new[3]], -1)
    _read_plain(st)


def _read_plain(st):
    for x, to in zip(_rows_of(st.case, st.cache[0][st.pages]), (st.k_out, st.v_out)):
        to.view(-1, *to.shape[2:])[st.rows_at] = x.transpose(1, 2).flatten(0, 1)[st.places_at].to(to.dtype)


def _pool_rows(c, pool):
    """K and V [..., 16, hd] of pages [..., 2, 16 * hd] of a context's pool."""
    hd, lead = c["hd"], pool.shape[:-2]
    k = pool[..., 0, :].reshape(lead + (hd // 8, PAGE, 8)).transpose(-2, -3).flatten(-2)
    v = pool[..., 1, :].reshape(lead + (hd // 16, 4, 16, 4)).movedim((-4, -3, -2, -1), (-2, -4, -1, -3)).flatten(-2)      # q, k, tile and n
    return k, v.flatten(-3, -2)


def _pool_pages(c, k, v):
    hd, lead = c["hd"], k.shape[:-2]
    k = k.reshape(lead + (PAGE, hd // 8, 8)).transpose(-2, -3).flatten(-3)
    v = v.reshape(lead + (4, 4, hd // 16, 16)).movedim((-4, -3, -2, -1), (-3, -1, -4, -2)).flatten(-4)      # tile, q, n, k
    return torch.stack([k, v], -2)


def _park_plain(st):
    """Whole pages in all layers at once; of a last page only the rows that there are."""
    c = st.case
    k, v = _pool_rows(c, st.pool[:, st.from_pages])                      # [layers, pages, heads, 16, hd]
    st.cache[:, st.pages] = _pages_of(c, torch.where(st.there, k, 0), torch.where(st.there, v, 0))
    _restore_plain(st)


def _restore_plain(st):
    c = st.case
    k, v = _rows_of(c, st.cache[:, st.pages])
    k0, v0 = _pool_rows(c, st.pool[:, st.to_pages])
    st.pool[:, st.to_pages] = _pool_pages(c, torch.where(st.there, k.to(k0.dtype), k0), torch.where(st.there, v.to(v0.dtype), v0))


# ---- from the definition, in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    st = _inputs(c, seed)
    return {"attend": _attend_exact, "store": _store_exact, "read": _read_exact, "park": _park_exact, "restore": _restore_exact}[c["op"]](c, st)


def _element(code, bits):
    """The number that a code of 4 or 8 bits stands for: (-1)^s (1 + m / 2^M) 2^(x - bias), without the 1 where x = 0."""
    M, X, bias = (1, 2, 1) if bits == 4 else (3, 4, 7)
    code = code.long()
    m, x, s = code & (1 << M) - 1, code >> M & (1 << X) - 1, code >> M + X
    one = (x > 0).double()
    return (1 - 2 * s).double() * (one + m.double() / 2 ** M) * torch.pow(torch.full((), 2.0, dtype=torch.float64, device=code.device), (x.clamp(min=1) - bias).double())


def _scale64(e):
    return torch.where(e.long() == 255, float("nan"), torch.pow(torch.full((), 2.0, dtype=torch.float64, device=e.device), e.double() - 127))


def _cached64(c, cache, layer, table_row, pos, head):
    """K and V of one head at positions `pos` of a sequence, [n, hd] in 64 bits, byte by byte from the layout."""
    nb, places = _blocks(c), _places(c)
    page, key = table_row.long()[pos // PAGE], (pos % PAGE)[:, None]
    flat = cache.view(-1)
    base = (((layer * cache.shape[1] + page) * cache.shape[2] + head) * cache.shape[3])[:, None]
    d = torch.arange(c["hd"], device=DEV)[None, :]
    b, i = d // 32, d % 32
    wide = torch.where(2 * (b // 2) + 2 <= nb, 2, 1)                # blocks that lie side by side, 8 bits
    out = []
    for part, bits in (("k", c["k_bits"]), ("v", c["v_bits"])):
        if part == "k":
            low = i % 2 == 0
            at = (b * 16 + key) * 16 + i // 2 if bits == 4 else ((i // 16 * nb + b) * 16 + key) * 16 + i % 16
        else:
            lane, low = key // 4 * 16 + i % 16, i < 16
            at = (lane * nb + b) * 4 + key % 4 if bits == 4 else b // 2 * 1024 + (lane * wide + b % 2) * 8 + key % 4 * 2 + i // 16
        code = flat[base + (places[0] if part == "k" else places[1]) + at]
        if bits == 4:
            code = torch.where(low, code & 15, code >> 4)
        e = flat[base + (places[2] if part == "k" else places[3]) + key * (4 if nb == 3 else nb) + b]
        out.append(_element(code, bits) * _scale64(e))
    return out


def _attend_exact(c, st):
    Hq, Hkv, hd = c["heads"], c["kv_heads"], c["hd"]
    G = Hq // Hkv
    out = torch.zeros(st.q.shape, dtype=torch.float64, device=DEV)
    for s, n_s in enumerate(st.lens):
        R = st.counts[s]
        n = n_s + R
        pos = torch.arange(n, device=DEV)
        for h in range(Hkv):
            K, V = _cached64(c, st.cache, 0, st.table[s], pos, h)
            q = st.q[s, :R, h * G:(h + 1) * G].double().reshape(R * G, hd)
            x = q @ K.T.contiguous() / hd ** 0.5
            if c["causal"]:
                x = torch.where(pos[None, :] <= n_s + torch.arange(R * G, device=DEV)[:, None] // G, x, -math.inf)
            out[s, :R, h * G:(h + 1) * G] = (torch.softmax(x, 1) @ V).view(R, G, hd)
    return out


def _held64(x, bits):
    """What rows [..., hd] become when they are held in `bits` bits."""
    hd = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -hd % 32)).unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    limit, largest, M, least = (7.0, 6.0, 1, 0) if bits == 4 else (464.0, 448.0, 3, -6)
    e = torch.full_like(most, -127.0)
    two = torch.full((), 2.0, dtype=torch.float64, device=x.device)
    guess = torch.where(most > 0, torch.floor(torch.log2(most / limit)) - 1, -127.0).clamp(min=-127.0)
    for _ in range(4):                                                # the least whole e with most / 2^e <= limit, the logarithm's rounding apart
        guess = torch.where(most / torch.pow(two, guess) > limit, guess + 1, guess)
    e = guess
    y = x / torch.pow(two, e)
    mag = torch.frexp(y)[1].double() - 1                              # floor of the binary logarithm
    step = torch.pow(two, torch.where(y == 0, least, mag).clamp(min=least) - M)
    y = (torch.round(y / step) * step).clamp(-largest, largest)       # torch.round: halves to even
    return (y * torch.pow(two, e)).flatten(-2)[..., :hd]


def _store_exact(c, st):
    out = []
    there = (torch.arange(c["rows"], device=DEV)[None, :] < st.counts_dev[:, None])[..., None, None]
    for x, bits in ((st.k, c["k_bits"]), (st.v, c["v_bits"])):
        out.append(torch.where(there, _held64(x, bits), 0.0))
    return out


def _read_exact(c, st):
    out = [torch.zeros(st.k_out.shape, dtype=torch.float64, device=DEV) for _ in range(2)]
    for s, n in enumerate(st.lens):
        R = st.counts[s]
        for h in range(c["kv_heads"] if R else 0):
            for to, x in zip(out, _cached64(c, st.cache, 0, st.table[s], torch.arange(n - R, n, device=DEV), h)):
                to[s, :R, h] = x
    return out


def _pool_at(c, pos):
    """Places of (K, V) of positions in a page's parts of the context's pool, [n, hd]."""
    key, d = (pos % PAGE)[:, None], torch.arange(c["hd"], device=DEV)[None, :]
    return d // 8 * 128 + key * 8 + d % 8, d // 16 * 256 + key // 4 * 64 + d % 16 * 4 + key % 4


def _park_exact(c, st):
    pool = st.pool
    out = pool.double()
    for s, n in enumerate(st.lens):
        pos = torch.arange(n, device=DEV)
        src, dst = st.from_table[s].long()[pos // PAGE], st.to_table[s].long()[pos // PAGE]
        for layer in range(c["layers"]):
            for part, (at, bits) in enumerate(zip(_pool_at(c, pos), (c["k_bits"], c["v_bits"]))):
                for h in range(c["kv_heads"]):
                    out[layer][dst[:, None], h, part, at] = _held64(pool[layer][src[:, None], h, part, at], bits)
    return out


def _restore_exact(c, st):
    out = st.pool.double()
    for s, n in enumerate(st.lens):
        pos = torch.arange(n, device=DEV)
        dst = st.to_table[s].long()[pos // PAGE]
        for layer in range(c["layers"]):
            for h in range(c["kv_heads"]):
                for part, (at, x) in enumerate(zip(_pool_at(c, pos), _cached64(c, st.cache, layer, st.table[s], pos, h))):
                    out[layer][dst[:, None], h, part, at] = x
    return out
