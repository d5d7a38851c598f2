"""Attention over caches in 4 and 8 bits where every key counts: ranges, wavefronts and pages that all carry weight, so that none of them can be lost or weighed wrongly unseen."""
import numpy as np
import pytest

from tests import kvq_model as km
from tests.shared_pages import PAGE
from tests.test_gpu_kvq import Setup, f64
from tests.test_gpu_kvq_numbers import _pair_bound

pytestmark = pytest.mark.gpu

WINDOW = 256   # keys: the least that a range has


def _even(x, q, K, lens, counts):
    """The largest share of a row's weight that a window of keys has, over the rows of sequences of more than four windows; of some rows."""
    most, group = 0.0, x.heads // x.kv
    for s, (n, c) in enumerate(zip(lens, counts)):
        if n <= 4 * WINDOW:
            continue
        for j in sorted({0, c // 2, c - 1}):
            pos = np.arange(n + j + 1)
            ids = x.table[s][pos // PAGE]
            there = (ids >= 0) & (ids < x.n_pages)
            for h in range(x.heads):
                score = np.einsum("kd,d->k", K[np.where(there, ids, 0), pos % PAGE, h // group], q[s, j, h]) / x.hd ** 0.5
                w = np.where(there, np.exp(score - score[there].max()), 0.0)
                most = max(most, np.add.reduceat(w, np.arange(0, len(w), WINDOW)).max() / w.sum())
    return most


def _run(x, q, lens, counts, hints, layer, causal=True):
    K, V = x.ref.rows(layer)
    ref, slack, wabs = km.attention64(f64(q), K, V, x.table, lens, counts, causal, x.n_pages)
    share = _even(x, f64(q), K, lens, counts)
    assert 0 < share < 0.7, share
    there = np.arange(q.shape[1])[None, :] < np.asarray(counts)[:, None]
    tol = np.maximum(_pair_bound(ref, slack, wabs, x.dtype), 1e-30)[there]
    outs = []
    for hint in hints:
        out = x.rows(q.shape)
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, layer, q, out, counts=x.ints(counts), causal=causal)
        x.e.device_status()
        over = np.abs(f64(out) - ref)[there] / tol
        assert over.max() <= 1, (hint, float(over.max()))
        again = out.clone().fill_(3.0)
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, layer, q, again, counts=x.ints(counts), causal=causal)
        assert x.torch.equal(again[x.dev(there)], out[x.dev(there)])
        outs.append(out)
    return outs


# few rows (eight times 32 lanes join a row's ranges) and many (32 lanes); tiles of 16, 32 and 64 rows
CUT = [("bf16", 8, 2, 128, (4, 4), 1, (3000, 5, 1027)), ("f32", 4, 2, 64, (8, 4), 1, (3000, 5, 1027)), ("bf16", 4, 1, 96, (8, 8), 3, (3000, 5, 1027)), ("f32", 2, 1, 128, (4, 8), 1, (20000, 7000)),
       ("bf16", 4, 4, 64, (8, 8), 1, (24000,)), ("f32", 32, 8, 32, (4, 4), 16, (2300, 700, 1100, 40, 0, 1999, 2000, 1500)), ("bf16", 32, 8, 64, (4, 8), 16, (2300, 700, 1100, 40, 0, 1999, 2000, 1500)),
       ("bf16", 32, 8, 128, (8, 4), 70, (1700, 2900)), ("f32", 4, 2, 48, (8, 8), 70, (3000, 5, 1027)), ("bf16", 10, 2, 80, (4, 4), 7, (5000, 1200)), ("bf16", 16, 2, 128, (8, 8), 40, (2500, 1300, 64, 9))]


@pytest.mark.parametrize("case", range(len(CUT)))
def test_cut_ranges_that_all_carry_weight(case):
    dtype, heads, kv, hd, bits, rows, lens = CUT[case]
    counts = tuple(max(1, rows - s) for s in range(len(lens)))
    x = Setup(dtype, heads, kv, hd, bits, len(lens), [n + rows for n in lens], seed=case, scales=(124, 128))
    x.poison(lens, counts)
    x.upload()
    q = x.rows((len(lens), rows, heads, hd), 0.4)
    _run(x, q, lens, counts, (max(lens), x.width * PAGE - 2, 0), 1)
    _run(x, q, lens, counts, (max(lens),), 0, causal=False)


@pytest.mark.parametrize("dtype,heads,kv,hd,bits,rows", [("bf16", 2, 1, 128, (4, 4), 1), ("bf16", 4, 2, 64, (8, 8), 9), ("bf16", 2, 1, 96, (4, 8), 33), ("f32", 2, 1, 32, (8, 4), 2),
                                                         ("f32", 2, 1, 128, (4, 8), 20)])
def test_long_ranges_whose_pages_all_carry_weight(dtype, heads, kv, hd, bits, rows):
    """Uncut (a hint of no tokens) and cut, more pages a wavefront than it asks the ids of at once, some missing in the middle."""
    lens, counts = (9100, 40), (rows, rows)
    x = Setup(dtype, heads, kv, hd, bits, 2, [n + rows for n in lens], seed=hd, scales=(124, 128))
    x.table[0, 77] = -1
    x.table[0, 300:304] = x.n_pages
    x.poison(lens, counts)
    x.upload()
    _run(x, x.rows((2, rows, heads, hd), 0.4), lens, counts, (0, 9100), 1)
