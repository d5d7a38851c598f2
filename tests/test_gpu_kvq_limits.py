"""Caches in 4 and 8 bits at the ends of what a call may say: hints, lengths and capacities."""
import numpy as np
import pytest

from tests import kvq_model as km
from tests.shared_pages import PAGE, dims
from tests.test_gpu_kvq import Setup, _check, _torch, f64

pytestmark = pytest.mark.gpu


class Pool:
    """A small context with something in its pool, a cache of sevens, and tables of pages for its sequences in both."""

    def __init__(self, dtype="bf16", seqs=2, width=4, block=2, hd=64, kv=2, bits=(4, 4)):
        import paper_2602_06036_amd as dfl
        from paper_2602_06036_amd import binding as B
        self.torch, self.B, self.width = _torch(), B, width
        self.n = seqs * width
        self.e = dfl.Engine(dims(1, 2 * kv, kv, hd), dims(1, 2 * kv, kv, hd), dtype, block, seqs, width, self.n, (0,), 63).create()
        self.data = self.torch.full((self.e.kvq_bytes(0, self.n, *bits),), 7, dtype=self.torch.uint8, device=self.e.device)
        self.cache = self.e.kvq(self.data, 0, self.n, *bits)
        pool = self.e.target_pool.view(self.torch.bfloat16 if dtype == "bf16" else self.torch.float32)
        g = self.torch.Generator(device=self.e.device)
        g.manual_seed(1)
        pool.copy_(self.torch.randn(pool.shape, generator=g, device=self.e.device))
        self.mine, self.theirs = (self.ints(np.random.RandomState(i).permutation(self.n).reshape(seqs, width)) for i in (0, 1))

    def ints(self, x):
        return self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device=self.e.device)

    def batch(self, lens, hint):
        self.lens = self.ints(lens)
        return self.e.batch(self.lens, self.mine, self.lens, hint)

    def status_is_capacity(self):
        with pytest.raises(self.B.DFlashError) as err:
            self.e.device_status()
        assert err.value.code == self.B.DFLASH_ECAPACITY


@pytest.mark.parametrize("lens", [[1, 0], [0, 40]])
def test_a_hint_of_no_tokens_does_not_lose_a_request_in_silence(lens):
    x = Pool()
    pool = x.e.target_pool.clone()
    for call in (x.B.dflash_kvq_pack, x.B.dflash_kvq_unpack):
        call(x.e, x.batch(lens, 0), x.cache, x.theirs)
        x.status_is_capacity()
    assert bool((x.data == 7).all()) and x.torch.equal(x.e.target_pool, pool)
    for call in (x.B.dflash_kvq_pack, x.B.dflash_kvq_unpack):       # nothing there, nothing said
        call(x.e, x.batch([0, 0], 0), x.cache, x.theirs)
    x.e.device_status()


@pytest.mark.parametrize("lens", [[-1, 20], [33, -(2 ** 31)]])
def test_negative_lengths_of_requests_raise_the_status(lens):
    x = Pool()
    for call in (x.B.dflash_kvq_pack, x.B.dflash_kvq_unpack):
        for hint in (0, 40):
            call(x.e, x.batch(lens, hint), x.cache, x.theirs)
            x.status_is_capacity()
    at = 0 if lens[0] < 0 else 1                              # such a sequence's pages stay as they are
    gone = x.theirs[at].long()
    assert bool((x.data.view(x.n, -1)[gone] == 7).all())


@pytest.mark.parametrize("lens,hint", [([-1, 20, 0], 20), ([500, 3, -7], 500), ([-(2 ** 31), 0, 700], 0)])
def test_negative_lengths_of_attention_count_as_none_and_raise_the_status(lens, hint):
    real = [max(n, 0) for n in lens]
    x = Setup("bf16", 4, 2, 64, (4, 8), 3, [n + 3 for n in real])
    x.poison(real, (3, 3, 3))
    x.upload()
    q, out = x.rows((3, 3, 4, 64)), x.rows((3, 3, 4, 64))
    before = out.clone()
    for counts in ((3, 3, 3), (1, 2, 3)):
        out.copy_(before)
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 0, q, out, counts=x.ints(counts))
        with pytest.raises(x.B.DFlashError) as err:
            x.e.device_status()
        assert err.value.code == x.B.DFLASH_ECAPACITY
        _check(x, q, out, before, real, counts, True, 0, (lens, counts))
    x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 0, q, out, counts=x.ints([0 if n < 0 else 1 for n in lens]))   # no rows of it, nothing to say
    x.e.device_status()


@pytest.mark.parametrize("rows,short", [(1, 1), (1, 0), (16, 16), (5, 4)])
def test_sequences_may_fill_their_block_table_row(rows, short):
    """The context's block of 16 rows means nothing to rows and attention: the last of them may be at the row's last position, under a hint that says so."""
    x = Setup("bf16", 4, 2, 64, (8, 4), 2, [40, 100], block=16, extra=4)
    spare = [p for p in range(x.n_pages) if p not in x.table]
    x.table[1, -2:] = spare[:2]
    cap = x.width * PAGE
    lens = [20, cap - short]
    counts = [rows, min(rows, short)]
    x.upload()
    b = x.batch(lens)
    k, v, q = x.rows((2, rows, 2, 64)), x.rows((2, rows, 2, 64)), x.rows((2, rows, 4, 64))
    c = x.ints(counts)
    x.B.dflash_kvq_write(x.e, b, x.cache, 1, k, v, counts=c)
    for s in range(2):
        for j in range(counts[s]):
            p = lens[s] + j
            x.ref.put(1, x.table[s, p // PAGE], p % PAGE, f64(k[s, j]), f64(v[s, j]))
    assert np.array_equal(x.data.cpu().numpy(), x.ref.data)
    ko, vo = x.torch.zeros_like(k), x.torch.zeros_like(v)
    x.B.dflash_kvq_read(x.e, b, x.cache, 1, ko, vo, x.lens_dev, counts=c)
    want = x.ref.rows(1)
    for s in range(2):
        for j in range(counts[s]):
            p = lens[s] + j
            for o, w in zip((ko, vo), want):
                assert np.array_equal(f64(o[s, j]), f64(x.torch.from_numpy(w[x.table[s, p // PAGE], p % PAGE]).to(x.tdt)))
    for causal in (True, False):
        out = x.rows(q.shape)
        before = out.clone()
        x.B.dflash_kvq_attention(x.e, b, x.cache, 1, q, out, counts=c, causal=causal)
        x.e.device_status()
        _check(x, q, out, before, lens, counts, causal, 1, (rows, short, causal))


@pytest.mark.parametrize("lens", [[64, 3], [48, 64], [49, 60]])
def test_requests_that_fill_their_block_table_row_are_put_aside_and_taken_up(lens):
    x = Pool(block=16, bits=(8, 8))
    before = x.e.target_pool.clone()
    b = x.batch(lens, max(lens))
    x.B.dflash_kvq_pack(x.e, b, x.cache, x.theirs)
    x.e.target_pool.zero_()
    x.B.dflash_kvq_unpack(x.e, b, x.cache, x.theirs)
    x.e.device_status()
    # [page, kv head, K | V, 16 rows of 64]: K [dim / 8][key][8], V [dim / 16][key / 4][dim % 16][key % 4]
    def rows(pool):
        p = pool.view(x.torch.bfloat16).view(x.n, 2, 2, 16 * 64).double().cpu()
        return p[:, :, 0].view(x.n, 2, 8, 16, 8).permute(0, 3, 1, 2, 4).reshape(x.n, 16, 2, 64), p[:, :, 1].view(x.n, 2, 4, 4, 16, 4).permute(0, 3, 5, 1, 2, 4).reshape(x.n, 16, 2, 64)
    table = x.mine.cpu().numpy()
    for old, new in zip(rows(before), rows(x.e.target_pool)):
        for s, n in enumerate(lens):
            for p in range(16 * x.width):
                a, w = new[table[s, p // PAGE], p % PAGE].numpy(), old[table[s, p // PAGE], p % PAGE].numpy()
                assert np.array_equal(a, km.values(*km.quantise(w, 8), 8, 64) if p < n else 0 * w), (s, p)


def test_hints_beyond_the_block_table_row_are_refused():
    import ctypes as C
    x = Pool(block=16)
    q = x.torch.zeros((2, 1, 4, 64), dtype=x.torch.bfloat16, device=x.e.device)
    out, k = q.clone(), q[:, :, :2].contiguous()
    b = x.batch([1, 1], 65)
    for call in (lambda: x.B.dflash_kvq_pack(x.e, b, x.cache, x.theirs), lambda: x.B.dflash_kvq_unpack(x.e, b, x.cache, x.theirs),
                 lambda: x.B.dflash_kvq_write(x.e, b, x.cache, 0, k, k), lambda: x.B.dflash_kvq_attention(x.e, b, x.cache, 0, q, out)):
        with pytest.raises(x.B.DFlashError) as err:
            call()
        assert err.value.code == x.B.DFLASH_ECAPACITY and "max_seq_len" in str(err.value)
    # neither anchors nor a block of the step's are looked at
    b = x.B.Batch(2, 20, x.lens.data_ptr(), x.theirs.data_ptr(), None, 99)
    x.B.dflash_kvq_attention(x.e, b, x.cache, 0, q, out)
    x.e.device_status()


@pytest.mark.parametrize("rows,lens,cut", [(1, [2000, 900, 40], True), (16, [30, 9, 0], False)])
def test_attention_launches_are_bracketed(rows, lens, cut):
    """dflash_profile_enable speaks of every attention launch: those of these calls, and the launches that join their ranges."""
    x = Setup("bf16", 8, 2, 64, (4, 8), 3, [n + rows for n in lens]).upload()
    q = x.rows((3, rows, 8, 64))
    out = x.torch.zeros_like(q)
    b = x.batch(lens)
    x.e.profile_enable(True)
    try:
        for _ in range(3):
            x.B.dflash_kvq_attention(x.e, b, x.cache, 1, q, out)
        prof = x.e.profile_read()
    finally:
        x.e.profile_enable(False)
    ms, n, read = prof[3]
    assert n == 3 and ms > 0
    assert read == 3 * 3 * (max(lens) + rows) * 2 * km.unit_bytes(64, 4, 8) / PAGE
    if cut:
        assert prof[4][1] == 3 and prof[4][0] > 0
    else:
        assert 4 not in prof
