"""Sequences that share pages on the GPU: the ledger's calls against the ledger kept in Python, attention of groups against 64 bits, and both in the step."""
from dataclasses import replace

import numpy as np
import pytest

from synth import inputs as si
from tests.helpers import W64, tiny_workload
from tests.shared_pages import PAGE, LedgerModel, allowed, attention64, dims, unpack

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _engine(dtype, target, draft, block, seqs, width, n_pages):
    import paper_2602_06036_amd as dfl
    e = dfl.Engine(target, draft, dtype, block, seqs, width, n_pages, (0,), 63).create()
    torch = _torch()
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pools = [p.view(tdt).view(m.n_layers, n_pages, m.n_kv_heads, 2, PAGE * m.head_dim) for p, m in ((e.target_pool, target), (e.draft_pool, draft))]
    return e, pools


# ---- attention ----------------------------------------------------------------------------------------------------------
LAYOUTS = [("f32", 4, 4, 64), ("f32", 6, 2, 48), ("f32", 2, 1, 128), ("f32", 3, 1, 16), ("bf16", 32, 8, 128), ("bf16", 8, 8, 64), ("bf16", 12, 4, 96),
           ("bf16", 16, 1, 32), ("bf16", 10, 2, 80), ("bf16", 8, 1, 128), ("bf16", 6, 2, 16), ("bf16", 4, 2, 112), ("bf16", 6, 2, 48)]
APART, ONCE = "1", "2"          # DFLASH_GROUP_APART: every sequence by itself; what a group shares once, by the plan, however small the call
# (rows, causal, lengths, pages shared by each group, group starts)
SHAPES = [
    (1, True, (0,), (0,), (0,)),                                        # one token, nothing cached
    (1, False, (33, 32, 47, 80), (2,), (0,)),                           # the shortest ends with the shared pages
    (2, True, (64, 64, 64), (4,), (0,)),                                # nothing but shared pages
    (3, True, (5, 0, 17, 16, 31), (0, 1), (0, 2)),                      # a sequence without tokens; a group whose sequences share nothing
    (7, False, (530, 515, 601, 40, 56), (32, 2), (0, 3)),
    (8, True, (150, 290, 170, 145, 160, 33, 35, 400), (9, 2, 0), (0, 5, 7)),   # the last group a single sequence
]


def _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, seed, layers=2):
    block = max(2, rows)
    S, rng = len(lens), np.random.RandomState(seed)
    width = max(lens) // PAGE + 3
    group = [max(g for g, a in enumerate(starts) if a <= s) for s in range(S)]
    held = [-(-(n + rows) // PAGE) for n in lens]
    n_pages = sum(shared) + sum(held) + 3
    ids = rng.permutation(n_pages).astype(np.int32)
    common, at = [], 0
    for x in shared:
        common.append(ids[at: at + x])
        at += x
    table = np.full((S, width), -1, np.int32)
    for s in range(S):
        k = min(shared[group[s]], held[s])
        table[s, :k] = common[group[s]][:k]
        table[s, k: held[s]] = ids[at: at + held[s] - k]
        at += held[s] - k
    m = dims(layers, heads, kv, hd)
    e, pools = _engine(dtype, m, m, block, S, width, n_pages)
    g = torch.Generator(device=e.device)
    g.manual_seed(seed)
    for p in pools:
        p.copy_(torch.randn(p.shape, generator=g, device=e.device))
    # rows that were never written and pages that nobody holds: anything
    for p in pools:
        k, v = unpack_index(torch, p, kv, hd)
        last = {}
        for s in range(S):
            for i in range(held[s]):
                last[int(table[s, i])] = max(last.get(int(table[s, i]), 0), min(PAGE, lens[s] + rows - PAGE * i))
        for page in range(n_pages):
            n = last.get(page, 0)
            k[:, page, n:] = float("nan")
            v[:, page, n:] = float("nan")
    q = (2 * torch.randn((S, rows, heads, hd), generator=g, device=e.device)).to(pools[0].dtype)
    return e, pools, table, n_pages, q


class unpack_index:
    """K and V of a pool by [layer, page, key from ..] for writing."""

    def __new__(cls, torch, pool, kv, hd):
        return _Rows(torch, pool, hd, 0), _Rows(torch, pool, hd, 1)


class _Rows:
    def __init__(self, torch, pool, hd, part):
        at = torch.arange(PAGE * hd, device=pool.device)
        self.pool, self.part, self.key = pool, part, (at // 8 % PAGE if part == 0 else at // 64 % 4 * 4 + at % 4)

    def __setitem__(self, where, value):
        layer, page, rows = where
        self.pool[layer, page, :, self.part, self.key >= rows.start] = value


def _attend(torch, e, table, lens, starts, q, pool, layer, causal, prefix_len):
    from paper_2602_06036_amd import binding as B
    dev = e.device
    t = torch.from_numpy(table).to(dev)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)
    st = torch.tensor(starts, dtype=torch.int32, device=dev)
    out = torch.full_like(q, 7.0)
    batch = e.batch(n, t, torch.zeros_like(n), max(lens))
    B.dflash_group_attention(e, batch, e.groups(st, prefix_len), pool, layer, q, out, causal=causal)
    torch.cuda.synchronize()
    return out


def _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, causal, dtype, kv, hd, prefix_len, pool=0, layer=1):
    got = _attend(torch, e, table, lens, starts, q, pool, layer, causal, prefix_len).double().cpu()
    k, v = (x.double().cpu() for x in unpack(pools[pool], layer, kv, hd))
    ref, slack, wabs = attention64(q.double().cpu(), k, v, table, lens, causal, n_pages)
    err, most = (got - ref).abs(), allowed(ref, slack, wabs, dtype)
    assert bool((err <= most).all()), (float((err - most).max()), float(err.max()))
    return got


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_attention_of_groups(layout, shape, way, monkeypatch):
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    dtype, heads, kv, hd = LAYOUTS[layout]
    rows, causal, lens, shared, starts = SHAPES[shape]
    rows = min(rows, 64 // (heads // kv))
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 100 * layout + shape)
    for hint in (max(shared) * PAGE, 0):          # the hint moves work between launches, not results
        _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, causal, dtype, kv, hd, hint, pool=shape % 2)
    e.device_status()
    e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd,rows,S,pages,own,causal", [
    ("bf16", 8, 2, 128, 16, 9, 65, 300, True), ("bf16", 8, 2, 128, 16, 9, 65, 300, False), ("bf16", 8, 1, 128, 16, 3, 130, 40, True),
    ("bf16", 4, 1, 128, 1, 40, 257, 20, True), ("bf16", 4, 4, 64, 5, 17, 33, 90, True), ("bf16", 2, 1, 128, 4, 2, 520, 1100, True),
    ("f32", 4, 1, 64, 8, 11, 40, 200, True), ("bf16", 4, 1, 128, 16, 1, 0, 700, True)])
def test_attention_over_long_contexts(dtype, heads, kv, hd, rows, S, pages, own, causal, monkeypatch):
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    lens = [pages * PAGE + (own * (i + 1)) // S + (i % 3) for i in range(S)]
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, (pages,), (0,), 5)
    _compare(torch, e, pools, table, lens, (0,), n_pages, q, rows, causal, dtype, kv, hd, pages * PAGE)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,hd,rows", [(12, 1, 64, 7), (40, 1, 128, 3), (32, 1, 128, 16), (64, 1, 64, 16), (24, 2, 128, 9)])
def test_more_than_64_rows_a_sequence(heads, kv, hd, rows, causal, way, monkeypatch):
    """Own parts of several tiles, whose borders fall between the heads of a slot."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    lens, shared, starts = (70, 83, 64, 0, 31), (4, 0), (0, 3)
    e, pools, table, n_pages, q = _case(torch, "bf16", heads, kv, hd, rows, lens, shared, starts, heads + rows)
    _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, causal, "bf16", kv, hd, 64)
    e.close()


@pytest.mark.parametrize("hd", [32, 64, 96, 128])
@pytest.mark.parametrize("pages", [1, 2, 3, 4, 5, 6, 7, 8, 9, 11, 12, 63, 64, 65, 67, 129, 131])
def test_tiles_over_prefix_lengths(hd, pages, monkeypatch):
    """One range of 1, 2, 3 .. pairs of pages, with and without a page B in the last one, and past the 32 pairs of a set of page ids."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    lens = [pages * PAGE + x for x in (3, 0, 19)]
    e, pools, table, n_pages, q = _case(torch, "bf16", 4, 1, hd, 16, lens, (pages,), (0,), 7 * pages + hd)
    _compare(torch, e, pools, table, lens, (0,), n_pages, q, 16, pages % 2 == 0, "bf16", 1, hd, 0)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 128), ("bf16", 64), ("bf16", 80)])
def test_scores_that_grow_and_keys_that_weigh_nothing(dtype, hd, way, monkeypatch):
    """Contexts whose scores grow by thousands from page to page (the reference maximum moves, what was there is scaled to nothing), or begin far below the others; keys at
    minus infinity weigh as if they were not there, also where they are all that a sweep has seen so far."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    rows, lens, shared, starts = 16, (160, 165, 190), (10,), (0,)
    e, pools, table, n_pages, q = _case(torch, dtype, 4, 1, hd, rows, lens, shared, starts, 11)
    saved = pools[0].clone()
    at = torch.arange(PAGE * hd, device=e.device)
    for factors in ((1, 2, 4, 8, 16, 32, 64, 128, 256, 512), (512, 64, 8, 1, 1, 1, 1, 1, 1, 1), (0.01,) * 8 + (100, 1)):
        for i, f in enumerate(factors):
            pools[0][1, int(table[0, i]), :, 0] = saved[1, int(table[0, i]), :, 0] * f
        _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, 1, hd, 160)
    # dim 0 of the queries is positive; the first three pages' keys are -inf there
    q[..., 0] = 1.0
    pools[0].copy_(saved)
    without = table.copy()
    without[:, :3] = -1
    _compare(torch, e, pools, without, lens, starts, n_pages, q, rows, True, dtype, 1, hd, 160)
    for i in range(3):
        pools[0][1, int(table[0, i]), :, 0, (at // 128 == 0) & (at % 8 == 0)] = float("-inf")
    got = _attend(torch, e, table, lens, starts, q, 0, 1, True, 160).double().cpu()
    k, v = (x.double().cpu() for x in unpack(saved, 1, 1, hd))
    want, slack, wabs = attention64(q.double().cpu(), k, v, without, lens, True, n_pages)
    assert bool(((got - want).abs() <= allowed(want, slack, wabs, dtype)).all()), float((got - want).abs().max())
    e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd,rows,lens", [("f32", 4, 4, 64, 8, (4000, 30)), ("bf16", 8, 2, 128, 16, (9000, 100, 3000))])
def test_a_long_context_by_itself(dtype, heads, kv, hd, rows, lens, monkeypatch):
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", APART)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, (0,), (0,), 6)
    _compare(torch, e, pools, table, lens, (0,), n_pages, q, rows, True, dtype, kv, hd, 0)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,heads,kv,hd", [("f32", 4, 2, 64), ("bf16", 4, 2, 128), ("bf16", 4, 2, 80), ("bf16", 64, 2, 64)])
def test_lengths_beyond_the_block_table(dtype, heads, kv, hd, way, monkeypatch):
    """Lengths on the device that no block-table row covers, up to the largest integer: the rows see every page of their block-table row and nothing else."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    from paper_2602_06036_amd import binding as B
    rows, lens, shared, starts = 2, (70, 84, 66, 20, 75), (4, 0), (0, 3)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 13)
    pools[0].copy_(torch.nan_to_num(pools[0], nan=0.5))          # pages that the longer lengths reach into
    cap, dev = table.shape[1] * PAGE, e.device
    for causal in (True, False):
        given = (2 ** 31 - 1, 84, 2 ** 31 - 1 - rows, cap - 1, cap + 3)
        t, n, out = torch.from_numpy(table).to(dev), torch.tensor(given, dtype=torch.int32, device=dev), torch.full_like(q, 7.0)
        B.dflash_group_attention(e, e.batch(n, t, torch.zeros_like(n), 84), e.groups(torch.tensor(starts, dtype=torch.int32, device=dev), 64), 0, 1, q, out, causal=causal)
        torch.cuda.synchronize()
        k, v = (x.double().cpu() for x in unpack(pools[0], 1, kv, hd))
        ref, slack, wabs = attention64(q.double().cpu(), k, v, table, given, causal, n_pages)
        assert bool(((out.double().cpu() - ref).abs() <= allowed(ref, slack, wabs, dtype)).all())
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,heads,kv,hd,rows", [("f32", 2, 2, 64, 1), ("bf16", 8, 2, 128, 4), ("bf16", 4, 2, 80, 3), ("bf16", 64, 2, 64, 4)])
def test_rows_beyond_the_block_table_raise_the_status(dtype, heads, kv, hd, rows, way, monkeypatch):
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    from paper_2602_06036_amd import binding as B
    lens, shared, starts = (40, 50), (2,), (0,)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 16)
    cap, dev = table.shape[1] * PAGE, e.device
    t, out = torch.from_numpy(table).to(dev), torch.empty_like(q)
    for last, fits in ((cap - rows, True), (cap - rows + 1, False), (2 ** 31 - 1, False), (50, True)):
        n = torch.tensor((40, last), dtype=torch.int32, device=dev)
        B.dflash_group_attention(e, e.batch(n, t, torch.zeros_like(n), 50), e.groups(None, 32), 0, 1, q, out)
        if fits:
            e.device_status()
        else:
            with pytest.raises(B.DFlashError) as err:
                e.device_status()
            assert err.value.code == B.DFLASH_ECAPACITY
    e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd", [("f32", 4, 4, 64), ("bf16", 8, 2, 128)])
def test_any_grouping_gives_the_same_rows(dtype, heads, kv, hd, monkeypatch):
    """Groups that do not match what is shared; starts that are not raise the status."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    from paper_2602_06036_amd import binding as B
    rows, lens, shared, starts = 4, (70, 80, 66, 90, 33, 40), (4, 2), (0, 4)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 3)
    for given, bad in (((0,), False), ((0, 1, 2, 3, 4, 5), False), ((0, 2, 3), False), ((0, 0, 3, 3), False), ((0, 5, 2), True), ((2, 3), True), ((0, 99), True),
                       ((0, -5, 4), True)):
        _compare(torch, e, pools, table, lens, given, n_pages, q, rows, True, dtype, kv, hd, 64)
        if bad:
            with pytest.raises(B.DFlashError) as err:
                e.device_status()
            assert err.value.code == B.DFLASH_ECAPACITY
        else:
            e.device_status()
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,heads,kv,hd", [("f32", 4, 2, 64), ("bf16", 4, 2, 128), ("bf16", 4, 2, 32), ("bf16", 4, 2, 80), ("bf16", 64, 2, 128)])
def test_missing_pages_and_nan_keys(dtype, heads, kv, hd, way, monkeypatch):
    """Entries outside the pool are keys that are not there, in the shared part of the table as behind it; a row without any is zeros; a NaN key
    makes the rows that see it NaN, and no others."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    rows, lens, shared, starts = 3 if heads < 64 else 2, (70, 84, 66, 20), (4, 0), (0, 3)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 4)
    table[:3, 2] = -1
    table[1, 4] = n_pages
    table[3, :] = -1
    got = _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, kv, hd, 64)
    assert (got[3] == 0).all()
    at = torch.arange(PAGE * hd, device=e.device)
    for page, key, hit in ((table[0, 1], 5, (0, 1, 2)), (table[2, 4], 3, (2,))):      # in the shared pages; the second row of sequence 2's block
        saved = pools[0].clone()
        pools[0][1, int(page), 0, 0, at // 8 % PAGE == key] = float("nan")            # kv head 0
        out = _attend(torch, e, table, lens, starts, q, 0, 1, True, 64).double().cpu()
        for s in range(4):
            for j in range(rows):
                sees = s in hit and (len(hit) == 3 or 4 * PAGE + key <= lens[s] + j)
                half = heads // kv
                assert torch.isnan(out[s, j, :half]).all() if sees else torch.equal(out[s, j, :half], got[s, j, :half]), (s, j)
                assert torch.equal(out[s, j, half:], got[s, j, half:])
        pools[0].copy_(saved)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,heads,kv,hd,rows", [("f32", 4, 2, 64, 12), ("f32", 4, 2, 128, 16), ("bf16", 4, 2, 128, 12), ("bf16", 4, 2, 32, 7), ("bf16", 4, 2, 80, 12),
                                                    ("bf16", 8, 2, 96, 16), ("bf16", 64, 2, 128, 2)])
def test_values_that_later_rows_see(dtype, heads, kv, hd, rows, way, monkeypatch):
    """V rows of the block itself with infinities and NaN: under the causal mask the rows in front of them are what they were, those behind get them in the dims that have
    them, and only there."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    lens, shared, starts = (70, 84, 64, 20, 127), (4, 0), (0, 3)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 6)
    got = _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, kv, hd, 64)
    planted = {s: s * 3 % rows for s in range(4)} | {4: rows - 1}          # sequence -> slot
    dims_of = ((0, hd - 1), (5, hd // 2))                                  # of kv head 0 and 1
    at = torch.arange(PAGE * hd, device=e.device)
    for s, slot in planted.items():
        pos = lens[s] + slot
        for h, bad in enumerate((float("nan"), float("-inf"))):
            for d in dims_of[h]:
                here = (at // (PAGE * 16) == d // 16) & (at // 64 % 4 == pos % PAGE // 4) & (at // 4 % 16 == d % 16) & (at % 4 == pos % 4)
                assert int(here.sum()) == 1
                pools[0][1, int(table[s, pos // PAGE]), h, 1, here] = bad
    k, v = (x.double().cpu() for x in unpack(pools[0], 1, kv, hd))
    out = _attend(torch, e, table, lens, starts, q, 0, 1, True, 64).double().cpu()
    half = heads // kv
    for s, slot in planted.items():
        pos = lens[s] + slot
        assert torch.isnan(v[table[s, pos // PAGE], pos % PAGE, 0, list(dims_of[0])]).all() and torch.isneginf(v[table[s, pos // PAGE], pos % PAGE, 1, list(dims_of[1])]).all()
        want = got[s].clone()
        for d in dims_of[0]:
            want[slot:, :half, d] = float("nan")
        for d in dims_of[1]:
            want[slot:, half: 2 * half, d] = float("-inf")
        assert torch.equal(torch.nan_to_num(out[s], nan=1e9), torch.nan_to_num(want, nan=1e9)), (s, slot)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,heads,kv,hd,rows", [("f32", 4, 2, 64, 12), ("bf16", 4, 2, 128, 12), ("bf16", 32, 2, 64, 4), ("bf16", 4, 2, 80, 12), ("bf16", 8, 2, 96, 1)])
def test_values_that_are_not_finite_under_any_grouping(dtype, heads, kv, hd, rows, causal, way, monkeypatch):
    """Infinities and NaN in V rows of committed keys, in the shared pages, behind them and next to the block, one of a key whose weight is 0 in fp32: the dims that have them
    are what the definition says, in the rows that see them, however the batch is cut; the other dims are what they were."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    lens, shared, starts = (170, 184, 164, 120, 127), (6, 3), (0, 3)
    e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, 15)
    q[..., 0] = 8.0
    at = torch.arange(PAGE * hd, device=e.device)

    def element(pos, d):
        return (at // (PAGE * 16) == d // 16) & (at // 64 % 4 == pos % PAGE // 4) & (at // 4 % 16 == d % 16) & (at % 4 == pos % 4)

    far = (at // 128 == 0) & (at % 8 == 0) & (at // 8 % PAGE == 7)            # dim 0 of K of the key 7 of a page
    pools[0][1, int(table[0, 2]), 0, 0, far] = -25.0 * hd ** 0.5              # its score: -200 and what the other dims give
    ways = [(starts, 96), (starts, 0), ((0,), 48), ((0, 1, 2, 3, 4), 160), ((0, 2, 3), 96)]
    before = [_compare(torch, e, pools, table, lens, g, n_pages, q, rows, causal, dtype, kv, hd, hint) for g, hint in ways]
    inf, nan = float("inf"), float("nan")
    #        sequence, position, dim, value: shared by 0 .. 2 (position < 96) or by 3 and 4 (< 48), else a sequence's own
    plants = [(0, 2 * PAGE + 7, 1, inf), (0, 5, hd - 1, -inf), (0, 70, 6, inf), (0, 71, 6, -inf), (3, 30, 2, nan), (1, 100, 3, inf), (2, 163, 4, -inf), (2, 161, 5, inf), (4, 126, 7, inf)]
    for s, pos, d, x in plants:
        pools[0][1, int(table[s, pos // PAGE]), 0, 1, element(pos, d)] = x
    want = {s: {} for s in range(5)}
    for s, pos, d, x in plants:
        for other in range(5):
            if table[other, pos // PAGE] == table[s, pos // PAGE]:
                want[other][d] = want[other].get(d, 0.0) + x
    k, v = (x.double().cpu() for x in unpack(pools[0], 1, kv, hd))
    ref, _, _ = attention64(q.double().cpu(), k, v, table, lens, causal, n_pages)
    half = heads // kv
    for (g, hint), old in zip(ways, before):
        out = _attend(torch, e, table, lens, g, q, 0, 1, causal, hint).double().cpu()
        for s in range(5):
            exp = old[s].clone()
            for d, x in want[s].items():
                exp[:, :half, d] = x
                assert torch.equal(torch.nan_to_num(ref[s, :, :half, d], nan=1e9), torch.nan_to_num(exp[:, :half, d], nan=1e9))
            assert torch.equal(torch.nan_to_num(out[s], nan=1e9), torch.nan_to_num(exp, nan=1e9)), (g, hint, s)
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 128), ("bf16", 64), ("bf16", 80)])
def test_large_values_behind_growing_scores(dtype, hd, way, monkeypatch):
    """Weights that outgrow the first page's by up to 2^50 meet values of 2^90: the sums stay finite, as the rows are."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    rows, lens, shared, starts = 16, (160, 165, 190), (10,), (0,)
    e, pools, table, n_pages, q = _case(torch, dtype, 4, 1, hd, rows, lens, shared, starts, 12)
    pools[0][1, :, :, 1] *= 2.0 ** 90
    for i in range(5, 10):
        pools[0][1, int(table[0, i]), :, 0] *= 6
    got = _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, 1, hd, 160)
    assert torch.isfinite(got).all()
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
@pytest.mark.parametrize("dtype,hd,key", [("bf16", 32, 7.75), ("bf16", 64, 11.0), ("bf16", 96, 13.375), ("bf16", 128, 15.5), ("bf16", 80, 12.25), ("f32", 64, 11.0)])
def test_large_values_behind_a_long_context(dtype, hd, key, way, monkeypatch):
    """One range of 513 pairs of pages whose first pair scores 15.8 powers of two below all others (8 * key / sqrt(hd) * log2 e): no pair is far above another, but together their
    weights pass 2^29, and meet values of 2^100: the sums stay finite, as the rows are."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    rows, pages, starts = 16, 1025, (0,)
    lens = (pages * PAGE + 3, pages * PAGE)
    assert 15.7 < 8 * key / hd ** 0.5 * 1.4427 < 16
    e, pools, table, n_pages, q = _case(torch, dtype, 4, 1, hd, rows, lens, (pages,), starts, 14)
    pools[0][1, :, :, 1] = pools[0][1, :, :, 1].abs() * 2.0 ** 100
    q.zero_()
    q[..., 0] = 8.0
    at = torch.arange(PAGE * hd, device=e.device)
    first = (at // 128 == 0) & (at % 8 == 0)                 # dim 0 of K
    for i in range(pages):
        pools[0][1, int(table[0, i]), :, 0, first] = 0.0 if i < 2 else key
    got = _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, 1, hd, 0)
    assert torch.isfinite(got).all()
    e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd,rows", [("f32", 2, 1, 16, 2), ("bf16", 4, 1, 32, 2), ("bf16", 2, 2, 48, 1)])
def test_many_sequences_and_groups(dtype, heads, kv, hd, rows, monkeypatch):
    """More sequences and more groups than a workgroup has threads, groups of no, one and many sequences."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    rng = np.random.RandomState(5)
    lens = tuple(int(x) for x in rng.randint(0, 60, size=300))
    for starts in (tuple([0, 0, 0] + sorted(int(x) for x in rng.randint(1, 300, size=277))), tuple(range(300)), (0, 290, 300)):
        shared = tuple(int(x) for x in rng.randint(0, 4, size=len(starts)))
        e, pools, table, n_pages, q = _case(torch, dtype, heads, kv, hd, rows, lens, shared, starts, len(starts))
        _compare(torch, e, pools, table, lens, starts, n_pages, q, rows, True, dtype, kv, hd, 32)
        e.device_status()
        e.close()


def test_two_graphs_share_a_workspace(monkeypatch):
    """Calls of different shapes captured into two graphs of one engine and replayed in turn, eager calls and the ledger's between them."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    from paper_2602_06036_amd import binding as B
    rows, lens, shared, starts = 8, (170, 180, 266, 190, 40), (10, 0), (0, 4)
    e, pools, table, n_pages, q = _case(torch, "bf16", 8, 2, 128, rows, lens, shared, starts, 9)
    dev = e.device
    t, n = torch.from_numpy(table).to(dev), torch.tensor(lens, dtype=torch.int32, device=dev)
    zero, two = torch.zeros_like(n), torch.tensor(starts, dtype=torch.int32, device=dev)
    refs = torch.from_numpy(np.bincount(table[table >= 0], minlength=n_pages).astype(np.int32)).to(dev)
    led, tokens = e.ledger(t, n, zero, refs), torch.zeros(5, dtype=torch.int32, device=dev)
    q3 = q[1:4, :1].contiguous()
    outs = [torch.zeros_like(q), torch.zeros_like(q3)]
    calls = [lambda out: B.dflash_group_attention(e, e.batch(n, t, zero, max(lens)), e.groups(two, 160), 0, 1, q, out),
             lambda out: B.dflash_group_attention(e, e.batch(n[1:4], t[1:4], zero[1:4], max(lens)), e.groups(None, 0), 1, 0, q3, out, causal=False)]
    graphs, side = [], torch.cuda.Stream()
    for call, out in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            call(out)
        graphs.append(g)
    for i in range(3):
        q.mul_(-1.0)
        q3.mul_(-1.0)
        want = []
        for call, out in zip(calls, outs):
            want.append(torch.zeros_like(out))
            call(want[-1])
            out.zero_()
        graphs[i % 2].replay()
        B.dflash_pages_reserve(e, led, tokens)
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out, w) and torch.isfinite(w).all()
    e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
def test_attention_on_a_stream_and_in_a_graph(way, monkeypatch):
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    from paper_2602_06036_amd import binding as B
    rows, lens, shared, starts = 4, (170, 180, 266, 190), (10,), (0,)
    e, pools, table, n_pages, q = _case(torch, "bf16", 8, 2, 128, rows, lens, shared, starts, 8)
    want = _attend(torch, e, table, lens, starts, q, 0, 1, True, 160)
    dev = e.device
    t, n, out = torch.from_numpy(table).to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), torch.zeros_like(q)
    batch, groups = e.batch(n, t, torch.zeros_like(n), max(lens)), e.groups(None, 160)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.dflash_group_attention(e, batch, groups, 0, 1, q, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.dflash_group_attention(e, batch, groups, 0, 1, q, out)
    other = q.clone()
    for i in range(4):
        q.copy_(other * (1 + i))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = torch.zeros_like(q)
        B.dflash_group_attention(e, batch, groups, 0, 1, q, again)
        torch.cuda.synchronize()
        assert torch.equal(out, again)
    e.close()


# ---- ledger -------------------------------------------------------------------------------------------------------------
class Pair:
    """An engine with its ledger, and the same in Python."""

    def __init__(self, torch, dtype, target, draft, rows, width, n_pages, max_seqs, seed=0):
        self.torch, self.t, self.d = torch, target, draft
        self.e, self.pools = _engine(dtype, target, draft, 4, max_seqs, width, n_pages)
        self.m = LedgerModel(rows, width, n_pages)
        dev = self.e.device
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        for p in self.pools:
            p.copy_(torch.randn(p.shape, generator=g, device=dev))
        self.host = [self._bits(p).cpu().clone() for p in self.pools]
        self.table, self.lens, self.anchor, self.refs = (torch.from_numpy(x.copy()).to(dev) for x in (self.m.table, self.m.lens, self.m.anchor, self.m.refs))
        self.l = self.e.ledger(self.table, self.lens, self.anchor, self.refs)

    def _bits(self, p):
        return p.view(self.torch.int16 if p.element_size() == 2 else self.torch.int32)

    def set_lens(self, lens):
        self.m.lens[: len(lens)] = lens
        self.m.anchor[: len(lens)] = np.arange(len(lens)) + 100
        self.push()

    def push(self):
        for dst, src in ((self.table, self.m.table), (self.lens, self.m.lens), (self.anchor, self.m.anchor), (self.refs, self.m.refs)):
            dst.copy_(self.torch.from_numpy(src))

    def check(self):
        self.torch.cuda.synchronize()
        for name in ("table", "lens", "anchor", "refs"):
            assert np.array_equal(getattr(self, name).cpu().numpy(), getattr(self.m, name)), name
        for i, (p, m) in enumerate(zip(self.pools, (self.t, self.d))):
            self.m.apply_copies(self.host[i], m.head_dim)
            assert self.torch.equal(self._bits(p).cpu(), self.host[i]), ("target", "draft")[i]
        self.m.copies = []
        counted = np.bincount(self.m.table[self.m.table >= 0], minlength=len(self.m.refs))
        assert np.array_equal(counted, self.m.refs)

    def reserve(self, tokens, status_ok=None):
        from paper_2602_06036_amd import binding as B
        want = self.m.reserve(tokens)
        dev = self.e.device
        granted = self.torch.full((len(tokens),), 9, dtype=self.torch.int32, device=dev)
        B.dflash_pages_reserve(self.e, self.l, self.torch.tensor(tokens, dtype=self.torch.int32, device=dev), granted)
        self.check()
        assert np.array_equal(granted.cpu().numpy(), want)
        if want.all():
            self.e.device_status()
        else:
            with pytest.raises(B.DFlashError) as err:
                self.e.device_status()
            assert err.value.code == B.DFLASH_ECAPACITY
        return want

    def fork(self, parents, children):
        from paper_2602_06036_amd import binding as B
        self.m.fork(parents, children)
        B.dflash_pages_fork(self.e, self.l, parents, children)
        self.check()

    def release(self, rows, keep=None):
        from paper_2602_06036_amd import binding as B
        self.m.release(rows, keep)
        B.dflash_pages_release(self.e, self.l, rows, keep)
        self.check()

    def compact(self):
        from paper_2602_06036_amd import binding as B
        n = self.m.compact()
        live = self.torch.zeros(1, dtype=self.torch.int32, device=self.e.device)
        B.dflash_pages_compact(self.e, self.l, live)
        self.check()
        assert int(live) == n
        assert (self.m.refs[:n] > 0).all() and (self.m.refs[n:] == 0).all()


MODELS = [("f32", dims(2, 4, 4, 64), dims(1, 4, 2, 64)), ("bf16", dims(3, 8, 2, 128), dims(1, 4, 1, 96)), ("bf16", dims(1, 2, 1, 16), dims(2, 6, 3, 80)),
          ("f32", dims(1, 2, 1, 16), dims(1, 3, 1, 48))]


@pytest.mark.parametrize("model", range(len(MODELS)))
def test_a_life_of_requests(model):
    """Prompts, samples of them, blocks written, samples dropped, holes closed: every call against the ledger in Python, every page of both pools bit for bit."""
    torch = _torch()
    dtype, t, d = MODELS[model]
    p = Pair(torch, dtype, t, d, 10, 9, 61, 8)
    p.reserve([37, 0, 100, 16, 1, -3])
    p.set_lens([37, 0, 100, 16, 1])
    p.fork([0, 2, 2, 3], [1, 5, 6, 7])
    p.reserve([8] * 8)                       # tails of 5 (two rows of 37), 4 (three of 100), a whole page (two of 16), and a page of its own
    p.reserve([8] * 8)                       # nothing left to ask for
    p.set_lens([45, 40, 108, 24, 9, 101, 104, 20])
    p.fork([5, 5, 0], [8, 9, 4])             # row 4 gives its pages back; rows 8 and 9 wait
    p.reserve([8] * 8)                       # rows 8 and 9 still hold row 5's tail: it gets a copy
    p.release([2, 7], [33, 0])
    p.compact()
    p.release([8])
    p.reserve([0, 12, 30, 0, 0, 5, 0, 7])
    p.fork([6], [8])
    p.release([0, 1, 2, 3, 4], [0, 16, 15, 17, 1000])
    p.compact()
    p.release(list(range(10)))
    p.compact()
    assert (p.m.refs == 0).all()
    p.e.close()


@pytest.mark.parametrize("tail", range(1, 16))
def test_copied_rows_of_a_tail(tail):
    torch = _torch()
    p = Pair(torch, "bf16", dims(2, 4, 2, 128), dims(1, 4, 1, 64), 4, 4, 16, 4)
    p.reserve([16 + tail])
    p.set_lens([16 + tail])
    p.fork([0, 0, 0], [1, 2, 3])
    assert p.reserve([1, 20, 0, 3]).all()
    p.e.close()


@pytest.mark.parametrize("way", [APART, ONCE])
def test_pages_beyond_four_gigabytes(way, monkeypatch):
    """A pool whose last pages lie more than 2^32 bytes (and 2^31 elements) behind its start: copied, moved and attended to."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    from paper_2602_06036_amd import binding as B
    m, n_pages = dims(40, 16, 8, 128), 2000
    e, pools = _engine("bf16", m, dims(1, 4, 1, 64), 4, 4, 6, n_pages)
    assert pools[0].numel() > 1 << 31
    dev, last = e.device, 39
    table = np.full((4, 6), -1, np.int32)
    table[0, :3], refs = [n_pages - 1, n_pages - 3, n_pages - 2], np.ones(n_pages, np.int32)     # everything in use but the pages below
    refs[[1990, 1995]] = 0
    g = torch.Generator(device=dev)
    g.manual_seed(2)
    for i in range(3):
        pools[0][last, n_pages - 1 - i].copy_(torch.randn(pools[0][last, 0].shape, generator=g, device=dev))
    t, n, a, r = (torch.from_numpy(x).to(dev) for x in (table, np.array([37, 0, 0, 0], np.int32), np.zeros(4, np.int32), refs))
    led = e.ledger(t, n, a, r)
    B.dflash_pages_fork(e, led, [0], [1])
    B.dflash_pages_reserve(e, led, torch.tensor([2, 2, 0, 0], dtype=torch.int32, device=dev))
    torch.cuda.synchronize()
    e.device_status()
    table[1] = table[0]
    table[0, 2] = 1990                                                  # the first to ask takes the copy, the last keeps the page
    assert np.array_equal(t.cpu().numpy(), table)
    k, v = (x.double().cpu() for x in unpack(pools[0], last, 8, 128))
    assert torch.equal(k[1990, :8], k[n_pages - 2, :8]) and torch.equal(v[1990, :8], v[n_pages - 2, :8]) and not k[1990, 8:].any()
    q = torch.randn((2, 2, 16, 128), generator=g, device=dev).bfloat16()
    for p in (1990, n_pages - 2):                                       # the two new rows of either sequence
        pools[0][last, p].copy_(torch.randn(pools[0][last, 0].shape, generator=g, device=dev))
    k, v = (x.double().cpu() for x in unpack(pools[0], last, 8, 128))
    ref, slack, wabs = attention64(q.double().cpu(), k, v, table, (37, 37), True, n_pages)
    out = _attend(torch, e, table[:2], (37, 37), (0,), q, 0, last, True, 32).double().cpu()
    assert bool(((out - ref).abs() <= allowed(ref, slack, wabs, "bf16")).all())
    r[:1000] = 0                                                        # holes: the high pages move down
    B.dflash_pages_compact(e, led)
    torch.cuda.synchronize()
    moved = t.cpu().numpy()
    assert (moved[:2, :3] < 1000).all() and (moved[2:] == -1).all()
    k2, _ = (x.double().cpu() for x in unpack(pools[0], last, 8, 128))
    for s in range(2):
        for i in range(3):
            assert torch.equal(k2[moved[s, i]], k[table[s, i]])
    e.close()


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 15, 5 * PAGE, 4 * PAGE + 1, 4 * PAGE, 0, -3])
def test_fork_of_any_length(length):
    """Lengths beyond the block-table row, up to the largest integer: all of its pages are shared, and the status says so."""
    torch = _torch()
    from paper_2602_06036_amd import binding as B
    p = Pair(torch, "f32", dims(1, 2, 1, 32), dims(1, 2, 1, 32), 3, 4, 12, 3)
    p.reserve([4 * PAGE, 20])
    p.set_lens([length, 20])
    p.fork([0], [2])
    if length > 4 * PAGE:
        with pytest.raises(B.DFlashError) as err:
            p.e.device_status()
        assert err.value.code == B.DFLASH_ECAPACITY
    else:
        p.e.device_status()
    p.e.close()


def test_too_few_pages_and_too_short_rows():
    torch = _torch()
    p = Pair(torch, "f32", dims(1, 2, 1, 32), dims(1, 2, 1, 32), 7, 6, 12, 6)
    assert list(p.reserve([40, 97, 30, 1, 0, 0])) == [1, 0, 1, 1, 1, 1]      # the second asks beyond its row
    p.set_lens([40, 0, 30, 1])
    p.fork([0, 0], [4, 5])
    # six pages left: row 0 takes a copy and one more, row 1 five (too many), and no row behind it takes any: rows 4 and 5 stay together
    assert list(p.reserve([20, 80, 2, 1, 3, 3])) == [1, 0, 1, 1, 0, 0]
    assert list(p.reserve([0, 0, 2, 1, 3, 0])) == [1, 1, 1, 1, 1, 1]
    p.release([1, 2, 3, 4, 5])
    assert list(p.reserve([0, 0, 0, 0, 96, 96])) == [1, 1, 1, 1, 1, 0]
    p.e.close()


def test_many_rows():
    """More rows than one launch takes: forks of 256, reservations of 1024."""
    torch = _torch()
    p = Pair(torch, "bf16", dims(1, 2, 1, 16), dims(1, 2, 1, 16), 1300, 3, 2700, 1200)
    p.reserve([20, 3])
    p.set_lens([20, 3])
    p.fork([i % 2 for i in range(1298)], list(range(2, 1300)))
    p.reserve([5] * 1200)                    # 98 waiting rows hold the tails too
    p.release(list(range(1299, 1, -1)), [4 + i % 20 for i in range(1298)])
    p.reserve([30] * 1200)
    p.compact()
    p.e.close()


def test_ledger_calls_in_a_graph():
    torch = _torch()
    from paper_2602_06036_amd import binding as B
    p = Pair(torch, "bf16", dims(2, 4, 2, 64), dims(1, 4, 2, 64), 6, 6, 40, 6)
    p.reserve([50])
    p.set_lens([50])
    parents, children = [0, 0, 0, 0], [2, 3, 4, 5]
    tokens = torch.full((6,), 8, dtype=torch.int32, device=p.e.device)
    tokens[1] = 0
    live = torch.zeros(1, dtype=torch.int32, device=p.e.device)

    def calls():
        B.dflash_pages_fork(p.e, p.l, parents, children)
        B.dflash_pages_reserve(p.e, p.l, tokens)
        B.dflash_pages_release(p.e, p.l, [3])
        B.dflash_pages_compact(p.e, p.l, live)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    torch.cuda.synchronize()
    p.check()                                # capturing ran nothing
    for i in range(4):
        p.m.fork(parents, children)
        p.m.reserve([8, 0, 8, 8, 8, 8])
        copies = list(p.m.copies)
        p.m.release([3])
        p.m.copies = copies
        for k, m in enumerate((p.t, p.d)):
            p.m.apply_copies(p.host[k], m.head_dim)
        n = p.m.compact()
        graph.replay()
        p.check()
        assert int(live) == n
        p.set_lens(p.m.lens.copy())          # eager work between replays
    p.e.close()


def test_refusals():
    torch = _torch()
    from paper_2602_06036_amd import binding as B
    p = Pair(torch, "f32", dims(2, 4, 2, 64), dims(1, 4, 4, 32), 5, 4, 20, 4)
    dev = p.e.device
    bad = [lambda: B.dflash_pages_fork(p.e, p.l, [0], [5]), lambda: B.dflash_pages_fork(p.e, p.l, [-1], [1]), lambda: B.dflash_pages_fork(p.e, p.l, [0, 0], [1, 1]),
           lambda: B.dflash_pages_fork(p.e, p.l, [0, 1], [1, 2]), lambda: B.dflash_pages_fork(p.e, p.l, [2], [2]),
           lambda: B.dflash_pages_release(p.e, p.l, [1, 1]), lambda: B.dflash_pages_release(p.e, p.l, [5]), lambda: B.dflash_pages_release(p.e, p.l, [1], [-1]),
           lambda: B.dflash_pages_reserve(p.e, p.l, torch.zeros(5, dtype=torch.int32, device=dev)),     # more than max_seqs
           lambda: B.dflash_pages_compact(p.e, B.Ledger(5, None, None, None, None)),
           lambda: B.dflash_pages_compact(p.e, B.Ledger(0, p.l.block_table, p.l.seq_lens, p.l.anchor, p.l.page_refs))]
    lens = torch.zeros(2, dtype=torch.int32, device=dev)
    batch, q = p.e.batch(lens, p.table[:2], lens, 10), torch.zeros((2, 3, 4, 64), device=dev)
    one = p.e.groups(None, 16)

    def attend(groups=one, pool=0, layer=0, q=q, out=None, batch=batch):
        return lambda: B.dflash_group_attention(p.e, batch, groups, pool, layer, q, torch.zeros_like(q) if out is None else out)

    starts = torch.zeros(3, dtype=torch.int32, device=dev)
    bad += [attend(groups=p.e.groups(starts, 0)), attend(groups=p.e.groups(None, -1)), attend(groups=B.Groups(2, 0, None)), attend(groups=B.Groups(0, 0, None)),
            attend(layer=2), attend(layer=-1), attend(q=torch.zeros((2, 5, 4, 64), device=dev)), attend(q=torch.zeros((2, 0, 4, 64), device=dev)),
            attend(q=torch.zeros(2 * 3 * 4 * 64 + 1, device=dev)[1:].view(2, 3, 4, 64)), attend(batch=p.e.batch(lens, p.table[:2], lens, 61)),
            lambda: B.dflash_set_groups(p.e, B.Groups(2, 0, None)), lambda: B.dflash_set_groups(p.e, p.e.groups(None, -2))]
    for i, call in enumerate(bad):
        with pytest.raises(B.DFlashError) as err:
            call()
        assert err.value.code in (B.DFLASH_EINVAL, B.DFLASH_ECAPACITY), i
        assert str(err.value), i
    for call in (attend(q=q.double()), attend(q=q[:1]), attend(q=q.transpose(1, 2)), attend(out=torch.zeros((2, 3, 4, 32), device=dev)),
                 attend(q=q.expand(2, 3, 4, 64).transpose(0, 1).transpose(0, 1)[:, :, :, ::2])):
        with pytest.raises((AssertionError, B.DFlashError)):
            call()
    p.check()                                # nothing happened
    # groups that do not fit a batch are refused by the step's calls, before anything is enqueued
    B.dflash_set_groups(p.e, p.e.groups(starts, 0))
    tok = torch.zeros((2, 4), dtype=torch.int32, device=dev)
    for call in (lambda: B.dflash_draft_block(p.e, batch, tok), lambda: B.dflash_verify(p.e, batch, tok, None)):
        with pytest.raises(B.DFlashError):
            call()
    p.e.device_status()
    p.e.close()


def test_groups_that_are_set_keep_their_starts():
    """The step's calls read the starts whenever they run: the tensor lives as long as the groups are set, and no longer; a refused call changes nothing."""
    torch = _torch()
    import gc
    import weakref
    from paper_2602_06036_amd import binding as B
    m = dims(1, 2, 1, 32)
    e, _ = _engine("f32", m, m, 4, 4, 4, 8)

    def given(n, prefix=0):
        starts = torch.arange(n, dtype=torch.int32, device=e.device)
        return e.groups(starts, prefix), weakref.ref(starts)

    def alive(ref):
        gc.collect()
        return ref() is not None

    g, first = given(2)
    B.dflash_set_groups(e, g)
    del g
    assert alive(first)
    g, other = given(3, -1)
    with pytest.raises(B.DFlashError):
        B.dflash_set_groups(e, g)
    del g
    assert alive(first) and not alive(other)
    g, second = given(3)
    B.dflash_set_groups(e, g)
    del g
    assert alive(second) and not alive(first)
    B.dflash_set_groups(e, None)
    assert not alive(second)
    e.close()


# ---- in the step --------------------------------------------------------------------------------------------------------
def _shared_model(w, wt, wd, prompts, children, steps):
    """A GpuModel whose sequences come out of prefilled prompts by forking; returns it with its ledger tensors."""
    torch = _torch()
    import paper_2602_06036_amd as dfl
    from tests.gpu_harness import GpuModel
    n = len(prompts) + sum(children)
    g = GpuModel(w, wt, wd, max(len(p) for p in prompts) + (steps + 2) * w.block_size, n_seqs=n)
    e, P = g.e, len(prompts)
    dev = e.device
    # order: every prompt, then its samples
    at, rows = [], 0
    for c in children:
        at.append(rows)
        rows += 1 + c
    table = torch.full((rows, e.max_pages_per_seq), -1, dtype=torch.int32, device=dev)
    lens, anchor = torch.zeros(rows, dtype=torch.int32, device=dev), torch.zeros(rows, dtype=torch.int32, device=dev)
    refs = torch.zeros(e.n_pages, dtype=torch.int32, device=dev)
    led = e.ledger(table, lens, anchor, refs)
    B = w.block_size
    ask = torch.zeros(rows, dtype=torch.int32)
    new = [0] * rows
    for a, p in zip(at, prompts):
        ask[a], new[a] = -(-len(p) // B) * B, len(p)
    dfl.dflash_pages_reserve(e, led, ask.to(dev))
    toks = torch.from_numpy(np.concatenate(prompts).astype(np.int32)).to(dev)
    dfl.dflash_prefill(e, e.batch(lens, table, anchor, 0), toks, new)
    parents = [a for a, c in zip(at, children) for _ in range(c)]
    kids = [a + 1 + i for a, c in zip(at, children) for i in range(c)]
    dfl.dflash_pages_fork(e, led, parents, kids)
    g.block_table, g.seq_lens, g.anchor, g.S = table, lens, anchor, rows
    owner = [i for i, c in enumerate(children) for _ in range(1 + c)]
    g.host_lens = np.array([len(prompts[i]) for i in owner], dtype=np.int64)
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    g.keep = (starts, refs)
    return g, led, e.groups(starts, min(len(p) for p in prompts) // PAGE * PAGE), owner


@pytest.mark.parametrize("way", [ONCE, "0"])
def test_forked_samples_step_as_the_oracle_does(way, monkeypatch):
    """fp32 model: two prompts, samples forked off them, then blocks drafted, verified, accepted and committed with the shared pages read once; the samples go
    different ways by their proposals.  Every sequence against the oracle's state of its own."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", way)
    from oracle import dflash_oracle as O
    import paper_2602_06036_amd as dfl
    w = tiny_workload(seed=9, n_layers=2, draft_layers=1, vocab=512, block=8, n_seqs=6, ctx=(60, 60), taps=(0,))
    wt, wd = si.make_weights(w, 4)
    Wt, Wd = W64(wt), W64(wd)
    prompts = [p[:n] for p, n in zip(si.make_prompts(w), (59, 38))]
    g, led, groups, owner = _shared_model(w, wt, wd, prompts, (3, 1), 5)
    dfl.dflash_set_groups(g.e, groups)
    states = []
    for i in owner:
        st = O.SeqState(w.target, w.draft, 59 + 6 * 8 + 1)
        O.prefill(Wt, Wd, w.target, w.draft, w.tap_layers, prompts[i], st)
        states.append(st)
    tokens = torch.full((6,), w.block_size, dtype=torch.int32, device=g.dev)
    granted = torch.zeros_like(tokens)
    rng = np.random.RandomState(1)
    for step in range(4):
        dfl.dflash_pages_reserve(g.e, led, tokens, granted)
        assert granted.all()
        # sample s keeps the first s of the target's own tokens, so that the samples commit different numbers
        prop = rng.randint(0, w.target.vocab - 1, size=(6, w.block_size - 1))
        for s in range(6):
            r = O.spec_step(Wt, Wd, w.target, w.draft, w.tap_layers, _copy(states[s]), w.block_size, w.mask_token_id, proposal=prop[s])
            for j in range(min(s, w.block_size - 1)):
                prop[s, j] = r["tgt_argmax"][j]
                r = O.spec_step(Wt, Wd, w.target, w.draft, w.tap_layers, _copy(states[s]), w.block_size, w.mask_token_id, proposal=prop[s])
        out = g.step(proposals=prop)
        for s in range(6):
            r = O.spec_step(Wt, Wd, w.target, w.draft, w.tap_layers, states[s], w.block_size, w.mask_token_id, proposal=prop[s])
            assert float(np.abs(out["logits_t"][s] - r["logits"]).max()) <= 1e-4
            assert int(out["accept_len"][s]) == r["accept_len"] and r["accept_len"] >= min(s, w.block_size - 1)
            assert list(out["out_tokens"][s, : r["accept_len"] + 1]) == r["emitted"]
    refs = g.keep[1].cpu().numpy()
    assert refs.max() == 4 and np.array_equal(np.bincount(g.block_table.cpu().numpy()[g.block_table.cpu().numpy() >= 0], minlength=len(refs)), refs)
    g.e.close()


def _copy(st):
    import copy
    return copy.deepcopy(st)


@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_bf16_step_with_and_without_groups(temperature, monkeypatch):
    """The same forked batch stepped with the groups set and without: either within the bf16 model's 2e-2 of exact order-free arithmetic (as the parity tests have it), so
    4e-2 apart at most; and without again, bit for bit."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    import paper_2602_06036_amd as dfl
    w = si.small_bf16_workload(n_seqs=7, ctx_min=20, ctx_max=150, seed=31, temperature=temperature)
    wt, wd = si.make_weights(w, 8)
    prompts = [np.resize(p, n) for p, n in zip(si.make_prompts(w), (149, 77))]
    g, led, groups, owner = _shared_model(w, wt, wd, prompts, (4, 1), 4)
    tokens = torch.full((7,), w.block_size, dtype=torch.int32, device=g.dev)
    dfl.dflash_pages_reserve(g.e, led, tokens)
    snap = [x.clone() for x in (g.e.target_pool, g.e.draft_pool, g.seq_lens, g.anchor)]
    lens = g.host_lens.copy()
    u = si.make_uniforms(w, 0) if temperature else None
    prop = np.random.RandomState(3).randint(0, w.target.vocab - 1, size=(7, w.block_size - 1))   # the same rows whatever the draft says

    def restore():
        for x, y in zip((g.e.target_pool, g.e.draft_pool, g.seq_lens, g.anchor), snap):
            x.copy_(y)
        g.host_lens = lens.copy()

    plain = g.step(proposals=prop, temperature=temperature, uniforms=u, key=5)
    restore()
    dfl.dflash_set_groups(g.e, groups)
    shared = g.step(proposals=prop, temperature=temperature, uniforms=u, key=5)
    for k in ("logits_d", "logits_t"):
        assert float(np.abs(plain[k] - shared[k]).max()) <= 4e-2, k
    # samples of one prompt see the same: their rows agree in both ways of computing
    for s in range(1, 5):
        assert np.array_equal(plain["logits_d"][0], plain["logits_d"][s])
    restore()
    dfl.dflash_set_groups(g.e, None)
    again = g.step(proposals=prop, temperature=temperature, uniforms=u, key=5)
    assert np.array_equal(again["logits_t"], plain["logits_t"])            # switched off: what it was
    g.e.close()
