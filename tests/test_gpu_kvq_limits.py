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
