"""Caches held in 4 or 8 bits on the GPU: rows written, read back, attended to, put aside and taken up again, against the format in numpy and attention in 64 bits."""
import numpy as np
import pytest

from tests import kvq_model as km
from tests.shared_pages import PAGE, dims, unpack

pytestmark = pytest.mark.gpu

BITS = [(4, 4), (8, 8), (8, 4), (4, 8)]


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


class Setup:
    """A context, a cache of random bytes with finite scales, and a block table of pages in random order."""

    def __init__(self, dtype, heads, kv, hd, bits, seqs, tokens, layers=2, pool_pages=1, block=2, extra=3, seed=0, scales=(118, 134)):
        import paper_2602_06036_amd as dfl
        from paper_2602_06036_amd import binding as B
        self.torch, self.B = _torch(), B
        self.tdt = self.torch.bfloat16 if dtype == "bf16" else self.torch.float32
        self.dtype, self.hd, self.bits, self.kv, self.heads = dtype, hd, bits, kv, heads
        self.rng = np.random.RandomState(seed)
        held = [-(-t // PAGE) for t in tokens]
        self.width, self.n_pages = max(held + [0]) + 2, sum(held) + extra
        self.e = dfl.Engine(dims(layers, heads, kv, hd), dims(1, heads, kv, hd), dtype, block, seqs, self.width, pool_pages, (0,), 63).create()
        ids = self.rng.permutation(self.n_pages).astype(np.int32)
        self.table, at = np.full((seqs, self.width), -1, np.int32), 0
        for s, h in enumerate(held):
            self.table[s, :h] = ids[at:at + h]
            at += h
        assert self.e.kvq_bytes(0, self.n_pages, *bits) == layers * self.n_pages * kv * km.unit_bytes(hd, *bits)
        data = self.rng.randint(0, 256, (layers, self.n_pages, kv, km.unit_bytes(hd, *bits))).astype(np.uint8)
        self.ref = km.Cache(data, hd, *bits)
        for part, b in enumerate(bits):
            if b == 8:                                      # no NaN codes: the format has none
                at = self.ref.at[part][0].ravel()
                x = data[..., at]
                data[..., at] = np.where(x & 127 == 127, x ^ 1, x)
            at = self.ref.at[2 + part].ravel()
            data[..., at] = self.rng.randint(*scales, data[..., at].shape) - (7 if b == 8 else 0)

    def upload(self):
        self.data = self.dev(self.ref.data)
        self.cache = self.e.kvq(self.data, 0, self.n_pages, *self.bits)
        return self

    def dev(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).to(self.e.device)

    def ints(self, x):
        return self.dev(np.asarray(x, np.int32))

    def batch(self, lens, hint=None, table=None):
        self.lens_dev, self.table_dev = self.ints(lens), self.ints(self.table if table is None else table)
        return self.e.batch(self.lens_dev, self.table_dev, self.torch.zeros_like(self.lens_dev), max(lens) if hint is None else hint)

    def rows(self, shape, scale=1.0):
        return self.dev(self.rng.standard_normal(shape) * scale).to(self.tdt)

    def poison(self, lens, counts):
        """Slots that no sequence holds: NaN scales, anything."""
        held = np.zeros((self.n_pages, PAGE), bool)
        for s, (n, c) in enumerate(zip(lens, counts)):
            for p in range(n + c):
                if 0 <= self.table[s, p // PAGE] < self.n_pages:
                    held[self.table[s, p // PAGE], p % PAGE] = True
        for part in (0, 1):
            at = self.ref.at[2 + part]
            for page in range(self.n_pages):
                for key in range(PAGE):
                    if not held[page, key]:
                        self.ref.data[:, page, :, at[key]] = 254 + (key + page) % 2


def f64(t):
    return t.double().cpu().numpy()


HDS = [("f32", 64), ("bf16", 128), ("bf16", 80), ("f32", 16), ("bf16", 32), ("f32", 112), ("bf16", 48), ("f32", 128), ("bf16", 64), ("bf16", 96)]


# ---- rows ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("dtype,hd", HDS)
def test_write_and_read(dtype, hd, bits):
    lens, counts, rows = [0, 5, 31, 16, 47, 3], [20, 20, 1, 0, 17, 12], 20
    x = Setup(dtype, 4, 2, hd, bits, 6, [n + rows for n in lens], seed=hd + bits[0]).upload()
    k, v = x.rows((6, rows, 2, hd)), x.rows((6, rows, 2, hd), 30.0)
    k[0, 3, 1] = 0
    k[1, 0, 0, 3] = float("inf")
    v[1, 2, 1, hd - 1] = float("nan")
    v[0, 7] *= 2.0 ** -100
    k[4, 5] *= 2.0 ** 100
    v[5, 1, 0, :8] = x.torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0])
    v[5, 1, 0, 8:] = 0
    b = x.batch(lens)
    c = x.ints(counts)
    x.B.dflash_kvq_write(x.e, b, x.cache, 1, k, v, counts=c)
    x.e.device_status()
    for s in range(6):
        for j in range(counts[s]):
            p = lens[s] + j
            x.ref.put(1, x.table[s, p // PAGE], p % PAGE, f64(k[s, j]), f64(v[s, j]))
    got = x.data.cpu().numpy()
    bad = np.argwhere(got != x.ref.data)
    assert not len(bad), (len(bad), bad[:5])
    # back, from other starts: rows of the sequences' middles, written and random ones
    starts, counts2 = [2, 0, 30, 7, 50, 3], [18, 11, 20, 0, 14, 1]
    ko, vo = x.rows((6, rows, 2, hd)), x.rows((6, rows, 2, hd))
    k0, v0 = ko.clone(), vo.clone()
    x.B.dflash_kvq_read(x.e, b, x.cache, 1, ko, vo, x.ints(starts), counts=x.ints(counts2))
    x.e.device_status()
    for part, (o, o0) in enumerate(((ko, k0), (vo, v0))):
        want = x.ref.rows(1)[part]
        for s in range(6):
            for j in range(rows):
                if j < counts2[s]:
                    p = starts[s] + j
                    w = x.torch.from_numpy(want[x.table[s, p // PAGE], p % PAGE]).to(x.tdt)
                    assert x.torch.equal(o[s, j].cpu().nan_to_num(12345.0), w.nan_to_num(12345.0)), (part, s, j)
                else:
                    assert x.torch.equal(o[s, j], o0[s, j])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [(4, 4), (8, 8)])
def test_extreme_rows(dtype, bits):
    """Every exponent that the type has, ties at every step, the smallest and the largest numbers."""
    x = Setup(dtype, 2, 1, 64, bits, 1, [300]).upload()
    n = 280
    vals = np.zeros((1, n, 1, 64))
    for j in range(n):
        vals[0, j, 0] = x.rng.choice([1.0, 1.75, 1.8125, 1.25, 1.5, 1.125, 1.9375, 1.0625], 64) * 2.0 ** np.clip(j - 150 - x.rng.randint(0, 12, 64).astype(float), -149, 127)
    k = x.dev(vals).to(x.tdt)
    v = -k
    b = x.batch([9])
    x.B.dflash_kvq_write(x.e, b, x.cache, 0, k, v)
    x.e.device_status()
    for j in range(n):
        x.ref.put(0, x.table[0, (9 + j) // PAGE], (9 + j) % PAGE, f64(k[0, j]), f64(v[0, j]))
    got = x.data.cpu().numpy()
    bad = np.argwhere(got != x.ref.data)
    assert not len(bad), (len(bad), bad[:5])


def test_written_rows_one_at_a_time_are_those_of_one_call():
    lens = [0, 13]
    a, b = (Setup("bf16", 4, 2, 128, (4, 8), 2, [n + 21 for n in lens], seed=5).upload() for _ in range(2))
    k, v = a.rows((2, 21, 2, 128)), a.rows((2, 21, 2, 128))
    a.B.dflash_kvq_write(a.e, a.batch(lens), a.cache, 1, k, v)
    for j in range(21):
        b.B.dflash_kvq_write(b.e, b.batch([n + j for n in lens]), b.cache, 1, k[:, j:j + 1].contiguous(), v[:, j:j + 1].contiguous())
    assert a.torch.equal(a.data, b.data)


# ---- attention ----------------------------------------------------------------------------------------------------------
LAYOUTS = [("bf16", 32, 8, 128), ("f32", 4, 4, 64), ("bf16", 8, 1, 64), ("f32", 6, 2, 48), ("bf16", 12, 4, 96), ("bf16", 10, 2, 80), ("f32", 2, 1, 128),
           ("bf16", 6, 2, 16), ("f32", 3, 1, 16), ("bf16", 4, 2, 112), ("bf16", 16, 1, 32), ("f32", 10, 1, 80)]
# (rows, causal, lengths, counts)
SHAPES = [
    (1, True, (0,), (1,)),
    (1, True, (1, 15, 16, 31, 32, 200), (1, 1, 0, 1, 1, 1)),
    (3, True, (0, 14, 45, 7), (3, 1, 2, 0)),
    (16, False, (130, 0, 63), (16, 5, 16)),
    (16, True, (500, 1, 48), (9, 16, 16)),
    (37, True, (0, 77, 300), (37, 20, 1)),
]


def _check(x, q, out, before, lens, counts, causal, layer, label):
    K, V = x.ref.rows(layer)
    ref, slack, wabs = km.attention64(f64(q), K, V, x.table, lens, counts, causal, x.n_pages)
    got, kept = f64(out), f64(before)
    for s in range(q.shape[0]):
        assert np.array_equal(got[s, counts[s]:], kept[s, counts[s]:]), (label, s)
    there = np.arange(q.shape[1])[None, :] < np.asarray(counts)[:, None]
    tol = km.allowed(ref, slack, wabs, x.dtype)[there]
    got, ref = got[there], ref[there]
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got), nan), (label, int((np.isnan(got) != nan).sum()))
    over = np.abs(got - ref)[~nan] / np.maximum(tol[~nan], 1e-30)
    assert not over.size or over.max() <= 1, (label, float(over.max()))


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
def test_attention(layout, shape):
    dtype, heads, kv, hd = LAYOUTS[layout]
    rows, causal, lens, counts = SHAPES[shape]
    for bits in BITS:
        x = Setup(dtype, heads, kv, hd, bits, len(lens), [n + c for n, c in zip(lens, counts)], seed=layout + 10 * shape)
        x.poison(lens, counts)
        x.upload()
        q, out = x.rows((len(lens), rows, heads, hd), 0.7), x.rows((len(lens), rows, heads, hd))
        before = out.clone()
        x.B.dflash_kvq_attention(x.e, x.batch(lens), x.cache, 1, q, out, counts=x.ints(counts), causal=causal)
        x.e.device_status()
        _check(x, q, out, before, lens, counts, causal, 1, (LAYOUTS[layout], SHAPES[shape], bits))


@pytest.mark.parametrize("dtype,heads,kv,hd,bits", [("bf16", 8, 2, 128, (4, 4)), ("f32", 4, 2, 64, (8, 4)), ("bf16", 4, 1, 96, (8, 8))])
@pytest.mark.parametrize("rows", [1, 70])
def test_attention_of_split_ranges(dtype, heads, kv, hd, bits, rows):
    """Long caches beside short ones, cut into ranges; a hint beyond the longest; counts left out; twice the same bits."""
    lens, counts = (3000, 5, 1027), (rows,) * 3
    x = Setup(dtype, heads, kv, hd, bits, 3, [n + rows for n in lens], seed=rows)
    x.poison(lens, counts)
    x.upload()
    q, out = x.rows((3, rows, heads, hd), 0.7), x.rows((3, rows, heads, hd))
    before = out.clone()
    for hint in (3000, x.width * PAGE - 2):
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 0, q, out)
        x.e.device_status()
        _check(x, q, out, before, lens, counts, True, 0, (dtype, hd, rows, hint))
        again = before.clone()
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 0, q, again)
        assert x.torch.equal(again, out)


@pytest.mark.parametrize("dtype,heads,kv,hd,bits,rows", [("bf16", 2, 1, 128, (4, 4), 1), ("bf16", 4, 2, 64, (8, 8), 9), ("bf16", 2, 1, 96, (4, 8), 33), ("f32", 2, 1, 32, (8, 4), 2),
                                                         ("f32", 2, 1, 128, (4, 8), 20)])
def test_attention_of_long_ranges(dtype, heads, kv, hd, bits, rows):
    """A hint of no tokens: nothing is cut, and a wavefront has more pages than it asks the ids of at once; a page is missing in the middle."""
    lens, counts = (9100, 40), (rows, rows)
    x = Setup(dtype, heads, kv, hd, bits, 2, [n + rows for n in lens], seed=hd)
    x.table[0, 77] = -1
    x.poison(lens, counts)
    x.upload()
    q, out = x.rows((2, rows, heads, hd), 0.7), x.rows((2, rows, heads, hd))
    before = out.clone()
    x.B.dflash_kvq_attention(x.e, x.batch(lens, 0), x.cache, 1, q, out)
    x.e.device_status()
    _check(x, q, out, before, lens, counts, True, 1, "long")


def test_attention_over_the_draft_and_many_sequences():
    """The draft's shape where it is another than the target's; more sequences than a wavefront has lanes, some without rows."""
    import paper_2602_06036_amd as dfl
    from paper_2602_06036_amd import binding as B
    torch = _torch()
    S, rng = 150, np.random.RandomState(0)
    lens = rng.randint(0, 90, S)
    lens[::40] = rng.randint(700, 1500, len(lens[::40]))
    counts = rng.randint(0, 3, S)
    held = -(-(lens + 2) // PAGE)
    width, n_pages = int(held.max()) + 1, int(held.sum())
    e = dfl.Engine(dims(2, 4, 2, 128), dims(3, 4, 1, 64), "bf16", 2, S, width, 1, (0,), 63).create()
    table, ids, at = np.full((S, width), -1, np.int32), rng.permutation(n_pages).astype(np.int32), 0
    for s in range(S):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    assert e.kvq_bytes(1, n_pages, 8, 4) == 3 * n_pages * km.unit_bytes(64, 8, 4)
    data = torch.zeros(e.kvq_bytes(1, n_pages, 8, 4), dtype=torch.uint8, device=e.device)
    cache = e.kvq(data, 1, n_pages, 8, 4)
    i32 = lambda t: torch.from_numpy(np.asarray(t, np.int32)).to(e.device)
    g = torch.Generator(device=e.device)
    g.manual_seed(3)
    rows = int(lens.max()) + 2
    k, v = (torch.randn((S, rows, 1, 64), generator=g, device=e.device).bfloat16() for _ in range(2))
    zero, table_dev, lens_dev, all_dev, counts_dev = i32(0 * lens), i32(table), i32(lens), i32(lens + counts), i32(counts)
    B.dflash_kvq_write(e, e.batch(zero, table_dev, zero, 0), cache, 2, k, v, counts=all_dev)
    q = torch.randn((S, 2, 4, 64), generator=g, device=e.device).bfloat16()
    for hint in (int(lens.max()), 90):
        out = torch.full_like(q, 7.0)
        before = out.clone()
        B.dflash_kvq_attention(e, e.batch(lens_dev, table_dev, zero, hint), cache, 2, q, out, counts=counts_dev, causal=False)
        e.device_status()
        ref = km.Cache(data.view(3, n_pages, 1, -1).cpu().numpy(), 64, 8, 4)
        exact, slack, wabs = km.attention64(f64(q), *ref.rows(2), table, lens, counts, False, n_pages)
        for s in range(S):
            c = counts[s]
            assert np.array_equal(f64(out)[s, c:], f64(before)[s, c:])
            assert (np.abs(f64(out)[s, :c] - exact[s, :c]) <= km.allowed(exact, slack, wabs, "bf16")[s, :c]).all(), s
    for bad in (k[..., :32], k):          # the draft's rows are 64 wide, the queries' heads four
        with pytest.raises(AssertionError):
            B.dflash_kvq_attention(e, e.batch(lens_dev, table_dev, zero, 90), cache, 2, bad.contiguous(), torch.zeros_like(bad.contiguous()))


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 48)])
def test_missing_pages_and_sequences_that_outgrow_the_table(dtype, hd):
    lens, counts, rows = [100, 70, 20, 0], [3, 3, 3, 3], 3
    x = Setup(dtype, 4, 2, hd, (4, 4), 4, [n + rows for n in lens])
    x.table[0, 2], x.table[0, 5], x.table[1, 0], x.table[1, 1] = -1, x.n_pages, -7, 1 << 30
    x.table[3, 0] = -1                                    # a row that sees no key
    x.poison(lens, counts)
    x.upload()
    q, out = x.rows((4, rows, 4, hd)), x.rows((4, rows, 4, hd))
    before = out.clone()
    x.B.dflash_kvq_attention(x.e, x.batch(lens), x.cache, 1, q, out, counts=x.ints(counts))
    x.e.device_status()
    _check(x, q, out, before, lens, counts, True, 1, "missing")
    # lengths that the hint or the table does not cover, counts beyond the rows: what there is, and the status
    cap = x.width * PAGE
    for lens2, counts2, hint in (([cap, 70, 20, 0], counts, 100), ([2 ** 31 - 1, 0, 0, -5], counts, 40), ([10, 10, 10, 10], [3, 4, 0, -1], 10)):
        out = before.clone()
        x.B.dflash_kvq_attention(x.e, x.batch(lens2, hint), x.cache, 1, q, out, counts=x.ints(counts2))
        with pytest.raises(x.B.DFlashError) as err:
            x.e.device_status()
        assert err.value.code == x.B.DFLASH_ECAPACITY
        if hint == 10:
            real = [3, 3, 0, 0]
            _check(x, q, out, before, lens2, real, True, 1, "counts")


def test_rows_outside_raise_the_status_and_write_nothing():
    x = Setup("bf16", 4, 2, 64, (4, 8), 3, [40, 40, 40]).upload()
    cap = x.width * PAGE
    x.table[1, 1] = -1
    k, v = x.rows((3, 20, 2, 64)), x.rows((3, 20, 2, 64))
    before = x.data.clone()
    for lens, counts in (([cap - 4, 0, 0], [20, 0, 0]), ([2 ** 31 - 3, 0, 0], [5, 0, 0]), ([0, 16, 0], [0, 4, 0]), ([0, 0, -3], [0, 0, 2])):
        x.data.copy_(before)
        b = x.batch(lens, 0)
        x.B.dflash_kvq_write(x.e, b, x.cache, 0, k, v, counts=x.ints(counts))
        with pytest.raises(x.B.DFlashError):
            x.e.device_status()
        assert x.torch.equal(x.data, before), (lens, counts)
        ko, vo = k.clone(), v.clone()
        x.B.dflash_kvq_read(x.e, b, x.cache, 0, ko, vo, x.ints(lens), counts=x.ints(counts))
        with pytest.raises(x.B.DFlashError):
            x.e.device_status()
        assert x.torch.equal(ko, k) and x.torch.equal(vo, v)
    # more rows than the call has: those it has
    b = x.batch([0, 0, 0], 0)
    x.B.dflash_kvq_write(x.e, b, x.cache, 0, k, v, counts=x.ints([0, 0, 21]))
    with pytest.raises(x.B.DFlashError):
        x.e.device_status()
    for j in range(20):
        x.ref.put(0, x.table[2, j // PAGE], j % PAGE, f64(k[2, j]), f64(v[2, j]))
    assert np.array_equal(x.data.cpu().numpy(), x.ref.data)


@pytest.mark.parametrize("dtype,heads,kv,hd,bits", [("bf16", 8, 2, 128, (4, 4)), ("f32", 4, 2, 64, (8, 8)), ("bf16", 4, 1, 48, (4, 8)), ("f32", 2, 2, 80, (4, 4))])
def test_nan_reaches_the_rows_that_see_it(dtype, heads, kv, hd, bits):
    lens, counts, rows = [30, 64, 9], [6, 6, 6], 6
    x = Setup(dtype, heads, kv, hd, bits, 3, [n + rows for n in lens])
    x.upload()
    k, v = x.rows((3, rows, kv, hd)), x.rows((3, rows, kv, hd))
    v[0, 3, 0, 1] = float("nan")                          # a block of the fourth row of the call
    k[1, 4, kv - 1, hd - 1] = float("inf")
    v[2, 5, 0, hd - 1] = float("-inf")
    b = x.batch(lens)
    x.B.dflash_kvq_write(x.e, b, x.cache, 0, k, v)
    for s in range(3):
        for j in range(rows):
            p = lens[s] + j
            x.ref.put(0, x.table[s, p // PAGE], p % PAGE, f64(k[s, j]), f64(v[s, j]))
    q, out = x.rows((3, rows, heads, hd)), x.rows((3, rows, heads, hd))
    for causal in (True, False):
        before = out.clone()
        x.B.dflash_kvq_attention(x.e, b, x.cache, 0, q, out, causal=causal)
        x.e.device_status()
        _check(x, q, out, before, lens, counts, causal, 0, causal)


def test_large_scores_and_values():
    """Scores of some thousands, a maximum that grows key by key, and values near the type's largest."""
    lens, counts = [190], [2]
    x = Setup("bf16", 2, 1, 64, (8, 8), 1, [192])
    x.upload()
    k = x.rows((1, 192, 1, 64)) + x.torch.arange(192, device=x.e.device).view(1, 192, 1, 1).to(x.tdt)
    v = x.rows((1, 192, 1, 64)) * 2.0 ** 118
    x.B.dflash_kvq_write(x.e, x.batch([0], 190), x.cache, 0, k, v)
    for j in range(192):
        x.ref.put(0, x.table[0, j // PAGE], j % PAGE, f64(k[0, j]), f64(v[0, j]))
    q = x.rows((1, 2, 2, 64)) + 1
    out = x.torch.zeros_like(q)
    x.B.dflash_kvq_attention(x.e, x.batch(lens), x.cache, 0, q, out)
    x.e.device_status()
    _check(x, q, out, out, lens, counts, True, 0, "large")


# ---- pages of the context's pool ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("pool", [0, 1])
@pytest.mark.parametrize("dtype,hd,bits", [("bf16", 128, (4, 4)), ("f32", 64, (8, 8)), ("bf16", 80, (8, 4)), ("f32", 16, (4, 8)), ("bf16", 48, (8, 8)), ("bf16", 96, (4, 4)),
                                           ("f32", 112, (4, 4)), ("bf16", 64, (4, 8))])
def test_pack_and_unpack(dtype, hd, bits, pool):
    import paper_2602_06036_amd as dfl
    from paper_2602_06036_amd import binding as B
    torch = _torch()
    lens = [0, 1, 16, 35, 63]
    S, kv, width, layers = len(lens), 2, 6, 3
    held = [-(-n // PAGE) for n in lens]
    pool_pages, n_pages = 2 * sum(held) + 2, sum(held) + 2
    m, d = dims(layers, 4, kv, hd), dims(2, 4, kv, hd)
    e = dfl.Engine(m, d, dtype, 2, S, width, pool_pages, (0,), 63).create()
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    mine, L = (e.target_pool, layers) if pool == 0 else (e.draft_pool, 2)
    mine = mine.view(tdt).view(L, pool_pages, kv, 2, PAGE * hd)
    g = torch.Generator(device=e.device)
    g.manual_seed(hd)
    mine.copy_(torch.randn(mine.shape, generator=g, device=e.device))
    rng = np.random.RandomState(hd)

    def tables(n, times):
        ids, out, at = rng.permutation(n).astype(np.int32), [], 0
        for _ in range(times):
            t = np.full((S, width), -1, np.int32)
            for s in range(S):
                t[s, :held[s]] = ids[at:at + held[s]]
                at += held[s]
            out.append(t)
        return out

    src, dst = tables(pool_pages, 2)
    (there,) = tables(n_pages, 1)
    # rows behind the sequences' ends, whatever they hold, are not put aside
    k, v = unpack(mine.double().cpu(), 0, kv, hd)
    k_all = [unpack(mine.double().cpu(), layer, kv, hd) for layer in range(L)]
    data = torch.from_numpy(rng.randint(0, 256, (L, n_pages, kv, km.unit_bytes(hd, *bits))).astype(np.uint8)).to(e.device)
    ref = km.Cache(data.cpu().numpy().copy(), hd, *bits)
    cache = e.kvq(data, pool, n_pages, *bits)
    dev = lambda t: torch.from_numpy(t).to(e.device)
    lens_dev = torch.tensor(lens, dtype=torch.int32, device=e.device)
    src_dev, dst_dev, there_dev = dev(src), dev(dst), dev(there)
    for s in range(S):
        if lens[s] % PAGE:                                      # beyond the last row: NaN in the pool
            page, n = int(src[s, held[s] - 1]), lens[s] % PAGE
            kk, vv = mine[:, page, :, 0].view(L, kv, hd // 8, PAGE, 8), mine[:, page, :, 1].view(L, kv, hd // 16, 4, 16, 4)
            kk[:, :, :, n:] = float("nan")
            for key in range(n, PAGE):
                vv[:, :, :, key // 4, :, key % 4] = float("nan")
    B.dflash_kvq_pack(e, e.batch(lens_dev, src_dev, lens_dev, max(lens)), cache, there_dev)
    e.device_status()
    for layer in range(L):
        k, v = (t.numpy() for t in k_all[layer])
        for s in range(S):
            for p in range(held[s] * PAGE):
                at, key = src[s, p // PAGE], p % PAGE
                zero = np.zeros((kv, hd))
                ref.put(layer, there[s, p // PAGE], key, k[at, key] if p < lens[s] else zero, v[at, key] if p < lens[s] else zero)
    got = data.cpu().numpy()
    nb = km.blocks(hd)
    if nb == 3:                                                 # the scales' fourth byte means nothing
        for x in (got, ref.data):
            end = km.unit_bytes(hd, *bits)
            x[..., np.arange(end - 128 + 3, end, 4)] = 0
    bad = np.argwhere(got != ref.data)
    assert not len(bad), (len(bad), bad[:5])
    before = mine.clone()
    B.dflash_kvq_unpack(e, e.batch(lens_dev, dst_dev, lens_dev, max(lens)), cache, there_dev)
    e.device_status()
    want = before.double().cpu()
    for layer in range(L):
        K, V = ref.rows(layer)
        wk = want[layer, :, :, 0].view(pool_pages, kv, hd // 8, PAGE, 8)
        wv = want[layer, :, :, 1].view(pool_pages, kv, hd // 16, 4, 16, 4)
        for s in range(S):
            for p in range(lens[s]):
                at, key, to = there[s, p // PAGE], p % PAGE, int(dst[s, p // PAGE])
                wk[to, :, :, key] = torch.from_numpy(K[at, key]).view(kv, hd // 8, 8)
                wv[to, :, :, key // 4, :, key % 4] = torch.from_numpy(V[at, key]).view(kv, hd // 16, 16)
    assert torch.equal(mine.cpu().nan_to_num(777.0), want.to(tdt).nan_to_num(777.0))


def test_pages_outside_are_not_packed():
    import paper_2602_06036_amd as dfl
    from paper_2602_06036_amd import binding as B
    torch = _torch()
    e = dfl.Engine(dims(1, 4, 2, 64), dims(1, 4, 2, 64), "bf16", 2, 2, 4, 4, (0,), 63).create()
    data = torch.full((e.kvq_bytes(0, 3, 4, 4),), 7, dtype=torch.uint8, device=e.device)
    cache = e.kvq(data, 0, 3, 4, 4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=e.device)
    lens, pool_before = i32([20, 33]), e.target_pool.clone()
    for mine, theirs, hint in (([[4, -1, -1, -1]] * 2, [[0, 1, 2, 0]] * 2, 33), ([[0, 1, 2, 3]] * 2, [[-1, 3, 1 << 30, -5]] * 2, 33)):
        mine, theirs = i32(mine), i32(theirs)
        b = e.batch(lens, mine, lens, hint)
        for call in (B.dflash_kvq_pack, B.dflash_kvq_unpack):
            call(e, b, cache, theirs)
            with pytest.raises(B.DFlashError):
                e.device_status()
    assert bool((data == 7).all()) and torch.equal(e.target_pool, pool_before)
    mine, theirs = i32([[0, 1, 2, 3]] * 2), i32([[0, 1, 2, 0], [1, 2, 0, 0]])
    B.dflash_kvq_pack(e, e.batch(lens, mine, lens, 16), cache, theirs)   # longer than the hint says
    with pytest.raises(B.DFlashError):
        e.device_status()


# ---- together -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,heads,kv,hd,bits", [("bf16", 32, 8, 128, (4, 4)), ("bf16", 8, 4, 64, (8, 8)), ("f32", 6, 2, 48, (8, 4))])
def test_a_request_put_aside_and_taken_up_again(dtype, heads, kv, hd, bits):
    """Cached rows packed, their pages given to others, unpacked elsewhere; new rows written to cache and pool: attention over the cache is attention over the restored pool."""
    import paper_2602_06036_amd as dfl
    from paper_2602_06036_amd import binding as B
    torch = _torch()
    lens, rows, S, width, layers = [210, 33, 64], 5, 3, 16, 2
    pool_pages = 64
    e = dfl.Engine(dims(layers, heads, kv, hd), dims(1, heads, kv, hd), dtype, 8, S, width, pool_pages, (0,), 63).create()
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pool = e.target_pool.view(tdt)
    g = torch.Generator(device=e.device)
    g.manual_seed(hd)
    pool.copy_(torch.randn(pool.shape, generator=g, device=e.device))
    ids = np.random.RandomState(1).permutation(pool_pages).astype(np.int32)
    held = [-(-(n + 8) // PAGE) for n in lens]
    tables = np.full((3, S, width), -1, np.int32)
    at = 0
    for t in (0, 1):
        for s in range(S):
            tables[t, s, :held[s]] = ids[at:at + held[s]]
            at += held[s]
    there = np.random.RandomState(2).permutation(sum(held)).astype(np.int32)
    for s, first in enumerate(np.cumsum([0] + held)[:S]):
        tables[2, s, :held[s]] = there[first:first + held[s]]
    old, new, there = (torch.from_numpy(t.copy()).to(e.device) for t in tables)
    lens_dev = torch.tensor(lens, dtype=torch.int32, device=e.device)
    data = torch.zeros(e.kvq_bytes(0, sum(held), *bits), dtype=torch.uint8, device=e.device)
    cache = e.kvq(data, 0, sum(held), *bits)
    before = [[B.dflash_kv_read(e, e.batch(lens_dev, old, lens_dev, max(lens)), 0, layer, s, 0, lens[s]) for s in range(S)] for layer in range(layers)]
    B.dflash_kvq_pack(e, e.batch(lens_dev, old, lens_dev, max(lens)), cache, there)
    pool.fill_(float("nan"))
    b = e.batch(lens_dev, new, lens_dev, max(lens))
    B.dflash_kvq_unpack(e, b, cache, there)
    q = torch.randn((S, rows, heads, hd), generator=g, device=e.device).to(tdt)
    k, v = (torch.randn((S, rows, kv, hd), generator=g, device=e.device).to(tdt) for _ in range(2))
    in_cache = e.batch(lens_dev, there, lens_dev, max(lens))
    for layer in range(layers):
        for s in range(S):                      # what came back is what the format makes of the rows
            for x, y, n in zip(before[layer][s], B.dflash_kv_read(e, b, 0, layer, s, 0, lens[s]), bits):
                w = torch.from_numpy(km.values(*km.quantise(x.double().cpu().numpy(), n), n, hd))
                assert torch.equal(y.cpu(), w.to(tdt).float())
        B.dflash_kvq_write(e, in_cache, cache, layer, k, v)
        kr, vr = torch.zeros_like(k), torch.zeros_like(v)
        B.dflash_kvq_read(e, in_cache, cache, layer, kr, vr, lens_dev)
        for s in range(S):
            B.dflash_kv_write(e, b, 0, layer, s, lens[s], kr[s].float(), vr[s].float())
        for causal in (True, False):
            out, want = torch.zeros_like(q), torch.zeros_like(q)
            B.dflash_kvq_attention(e, in_cache, cache, layer, q, out, causal=causal)
            B.dflash_group_attention(e, b, e.groups(torch.arange(S, dtype=torch.int32, device=e.device), 0), 0, layer, q, want, causal=causal)
            # each within its own bound of exact arithmetic
            ref = km.Cache(data.view(layers, sum(held), kv, -1).cpu().numpy(), hd, *bits)
            exact, slack, wabs = km.attention64(f64(q), *ref.rows(layer), tables[2], lens, [rows] * S, causal, sum(held))
            tol = km.allowed(exact, slack, wabs, dtype)
            assert (np.abs(f64(out) - exact) <= tol).all() and (np.abs(f64(want) - exact) <= tol).all()
    e.device_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed_on_another_stream(dtype):
    lens, rows = [700, 33, 1500], 2
    x = Setup(dtype, 8, 2, 64, (8, 4), 3, [n + 40 for n in lens]).upload()
    torch, B = x.torch, x.B
    k, v = x.rows((3, rows, 2, 64)), x.rows((3, rows, 2, 64))
    q = x.rows((3, rows, 8, 64))
    b, b2 = x.batch(lens, max(lens) + 30), None
    lens_dev = x.lens_dev
    outs = [torch.zeros_like(q) for _ in range(2)]
    kr, vr = torch.zeros_like(k), torch.zeros_like(v)

    def go(out, causal):
        B.dflash_kvq_write(x.e, b, x.cache, 1, k, v)
        B.dflash_kvq_attention(x.e, b, x.cache, 1, q, out, causal=causal)
        B.dflash_kvq_read(x.e, b, x.cache, 1, kr, vr, lens_dev)

    go(outs[0], True)
    go(outs[1], False)
    torch.cuda.synchronize()
    graphs = []
    for i, causal in enumerate((True, False)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(outs[i], causal)
        graphs.append(g)
    other = torch.cuda.Stream()
    for turn in range(3):
        torch.manual_seed(turn)
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape))
        lens_dev += 5
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs] + [kr.clone(), vr.clone()]
        go(outs[0], True)
        go(outs[1], False)
        torch.cuda.synchronize()
        for a, w in zip(got, outs + [kr, vr]):
            assert torch.equal(a, w), turn
    x.e.device_status()


def test_cache_beyond_4_gb():
    """Pages whose bytes lie behind 2^32."""
    import paper_2602_06036_amd as dfl
    from paper_2602_06036_amd import binding as B
    torch = _torch()
    hd, kv, n_pages, width = 128, 8, 300000, 8
    e = dfl.Engine(dims(1, 32, kv, hd), dims(1, 32, kv, hd), "bf16", 2, 2, width, 1, (0,), 63).create()
    data = torch.zeros(e.kvq_bytes(0, n_pages, 4, 4), dtype=torch.uint8, device=e.device)
    assert data.numel() > 2 ** 32
    cache = e.kvq(data, 0, n_pages, 4, 4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=e.device)
    outs = []
    for first in (0, n_pages - 16):
        table = i32([[first + 2 * i + s for i in range(width)] for s in range(2)])
        g = torch.Generator(device=e.device)
        g.manual_seed(1)
        k, v = (torch.randn((2, 100, kv, hd), generator=g, device=e.device).bfloat16() for _ in range(2))
        q = torch.randn((2, 3, 32, hd), generator=g, device=e.device).bfloat16()
        zero, lens = i32([0, 0]), i32([97, 60])
        B.dflash_kvq_write(e, e.batch(zero, table, zero, 0), cache, 0, k, v)
        out, kr, vr = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        B.dflash_kvq_attention(e, e.batch(lens, table, zero, 97), cache, 0, q, out)
        B.dflash_kvq_read(e, e.batch(lens, table, zero, 97), cache, 0, kr, vr, zero)
        outs.append((out, kr, vr))
    e.device_status()
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert float(outs[0][0].abs().max()) > 0 and float(outs[0][1].abs().max()) > 0


# ---- refusals ------------------------------------------------------------------------------------------------------------------
def test_refusals():
    import ctypes as C
    x = Setup("bf16", 4, 2, 64, (4, 4), 2, [40, 40]).upload()
    torch, B, e = x.torch, x.B, x.e
    b = x.batch([10, 20])
    q, k = x.rows((2, 3, 4, 64)), x.rows((2, 3, 2, 64))
    out, table = torch.zeros_like(q), x.ints(x.table)
    P = lambda t: t.data_ptr()

    def refused(code, word, rc):
        msg = e.l.dflash_last_error(e.ctx).decode()
        assert rc == code and word in msg, (rc, msg)

    def cache(**kw):
        c = e.kvq(x.data, 0, x.n_pages, 4, 4)
        for n, val in kw.items():
            setattr(c, n, val)
        return c

    def each(c, layer=0, rows=3):
        yield e.l.dflash_kvq_write(e.ctx, C.byref(b), C.byref(c), layer, rows, None, P(k), P(k), None)
        yield e.l.dflash_kvq_read(e.ctx, C.byref(b), C.byref(c), layer, rows, P(x.lens_dev), None, P(k), P(q), None)
        yield e.l.dflash_kvq_attention(e.ctx, C.byref(b), C.byref(c), layer, rows, None, 1, P(q), P(out), None)

    def pages(c):
        yield e.l.dflash_kvq_pack(e.ctx, C.byref(b), C.byref(c), P(table), None)
        yield e.l.dflash_kvq_unpack(e.ctx, C.byref(b), C.byref(c), P(table), None)

    E, W, K = B.DFLASH_EINVAL, B.DFLASH_EWORKSPACE, B.DFLASH_ECAPACITY
    for kw, code, word in ((dict(data=None), E, "null cache"), (dict(pool=2), E, "pool"), (dict(k_bits=5), E, "bits"), (dict(v_bits=16), E, "bits"), (dict(n_pages=0), E, "pages"),
                           (dict(data=P(x.data) + 16), E, "aligned"), (dict(bytes=x.data.numel() - 1), W, "bytes"), (dict(n_pages=x.n_pages + 1), W, "bytes"),
                           (dict(k_bits=8), W, "bytes")):
        for calls in (each, pages):
            for rc in calls(cache(**kw)):
                refused(code, word, rc)
    for kw, code, word in ((dict(layer=-1), E, "layer"), (dict(layer=2), E, "layer"), (dict(rows=0), E, "rows"), (dict(rows=x.width * PAGE + 1), K, "rows")):
        for rc in each(cache(), **kw):
            refused(code, word, rc)
    c = cache()
    refused(E, "aligned", e.l.dflash_kvq_attention(e.ctx, C.byref(b), C.byref(c), 0, 3, None, 1, P(q) + 2, P(out), None))
    refused(E, "overlap", e.l.dflash_kvq_attention(e.ctx, C.byref(b), C.byref(c), 0, 3, None, 1, P(q), P(q), None))
    refused(E, "overlap", e.l.dflash_kvq_attention(e.ctx, C.byref(b), C.byref(c), 0, 3, None, 1, P(q), P(q) + q.numel() * 2 - 16, None))
    refused(E, "overlap", e.l.dflash_kvq_read(e.ctx, C.byref(b), C.byref(c), 0, 3, P(x.lens_dev), None, P(k), P(k), None))
    refused(E, "aligned", e.l.dflash_kvq_attention(e.ctx, C.byref(b), C.byref(c), 0, 3, None, 1, None, P(out), None))
    refused(E, "aligned", e.l.dflash_kvq_write(e.ctx, C.byref(b), C.byref(c), 0, 3, None, P(k), None, None))
    refused(E, "starts", e.l.dflash_kvq_read(e.ctx, C.byref(b), C.byref(c), 0, 3, None, None, P(k), P(k), None))
    refused(E, "table", e.l.dflash_kvq_pack(e.ctx, C.byref(b), C.byref(c), None, None))
    refused(E, "null cache", e.l.dflash_kvq_pack(e.ctx, C.byref(b), None, P(table), None))
    bad = B.Batch(3, 10, b.seq_lens, b.block_table, b.anchor, 0)
    refused(E, "n_seqs", e.l.dflash_kvq_attention(e.ctx, C.byref(bad), C.byref(c), 0, 3, None, 1, P(q), P(out), None))
    none = B.Batch(0, 0, None, None, None, 0)
    assert e.l.dflash_kvq_attention(e.ctx, C.byref(none), C.byref(c), 0, 3, None, 1, None, None, None) == B.DFLASH_OK
    for args in ((q[:, :, :2].contiguous(), out), (q.float(), out.float()), (q[:1], out[:1])):
        with pytest.raises(AssertionError):
            B.dflash_kvq_attention(e, b, c, 0, *args)
    with pytest.raises(AssertionError):
        B.dflash_kvq_attention(e, b, c, 0, q, out, counts=torch.zeros(2, dtype=torch.int64, device=e.device))
    with pytest.raises(B.DFlashError):
        e.kvq_bytes(0, 4, 4, 5)
    e.device_status()
