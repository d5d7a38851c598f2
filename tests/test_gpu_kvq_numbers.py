"""What attention over caches in 4 and 8 bits makes of numbers at the ends of their range, and of weights that many keys share, against attention in 64 bits."""
import numpy as np
import pytest

from tests import kvq_model as km
from tests.shared_pages import PAGE
from tests.test_gpu_kvq import Setup, _check, f64

pytestmark = pytest.mark.gpu


def _scales(x, part, e):
    """All scales of K (part 0) or V; e as for 4-bit codes, so that the largest value is 6 * 2^(e - 127) in 4 bits and 7 * 2^(e - 127) in 8."""
    x.ref.data[..., x.ref.at[2 + part].ravel()] = e - (6 if x.bits[part] == 8 else 0)


# heads, kv heads, head dim, bits, rows, lengths: tiles of 16, 32 and 64 rows, whole and cut ranges, both forms of the merge
NUMBERS = [("bf16", 4, 1, 128, (4, 4), 1, (300, 3000, 0)), ("bf16", 8, 2, 64, (8, 8), 5, (40, 1)), ("bf16", 32, 8, 128, (8, 4), 70, (1500, 700)), ("bf16", 4, 1, 96, (4, 8), 6, (2500, 31)),
           ("f32", 4, 2, 64, (8, 8), 1, (300, 3000, 0)), ("f32", 8, 2, 128, (4, 4), 7, (40, 2200)), ("f32", 32, 2, 32, (4, 8), 70, (1500, 900)), ("bf16", 2, 1, 80, (8, 8), 1, (9000,))]


@pytest.mark.parametrize("v_scale", [252, 20])
@pytest.mark.parametrize("case", range(len(NUMBERS)))
def test_weighted_means_of_the_largest_and_smallest_values(case, v_scale):
    """Keys with about the same weight: the sum of their values is beyond the type, their mean is not (up to 1.75 * 2^127; one block of a head has the largest code everywhere).
    Values of 2^-107 keep their bits all the same."""
    dtype, heads, kv, hd, bits, rows, lens = NUMBERS[case]
    counts = (rows,) * len(lens)
    x = Setup(dtype, heads, kv, hd, bits, len(lens), [n + rows for n in lens], seed=case)
    _scales(x, 0, 112)                          # scores of some hundredths: hundreds of keys of each row weigh about the same
    _scales(x, 1, v_scale)
    x.ref.data[:, :, 0, x.ref.at[1][0][:, 0].ravel()] = 0x77 if bits[1] == 4 else 0x7E
    x.poison(lens, counts)
    x.upload()
    q, out = x.rows((len(lens), rows, heads, hd), 0.7), x.rows((len(lens), rows, heads, hd))
    before = out.clone()
    for hint, causal in ((max(lens), True), (0, False)):
        out.copy_(before)
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 1, q, out, causal=causal)
        x.e.device_status()
        assert bool(x.torch.isfinite(out).all()), (case, v_scale, hint)
        _check(x, q, out, before, lens, counts, causal, 1, (case, v_scale, hint))


# power of two of the scores' size; below 2^30 is ordinary ground
@pytest.mark.parametrize("power", [20, 31, 34, 60, 100])
@pytest.mark.parametrize("dtype,heads,kv,hd,bits,rows,lens", [("bf16", 4, 1, 64, (4, 4), 1, (200, 2600)), ("f32", 4, 2, 16, (8, 4), 3, (70, 1900)), ("bf16", 32, 8, 64, (4, 8), 40, (900, 33)),
                                                              ("f32", 2, 1, 64, (4, 4), 20, (2300,))])
def test_very_large_scores(dtype, heads, kv, hd, bits, rows, lens, power):
    """q has one dim, so scores are one product and exact, positive for a row of heads and negative for the next: a row is the mean of the keys that share its largest."""
    counts = (rows,) * len(lens)
    x = Setup(dtype, heads, kv, hd, bits, len(lens), [n + rows for n in lens], seed=power)
    _scales(x, 0, 127 + power // 2)
    _scales(x, 1, 127)
    x.poison(lens, counts)
    x.upload()
    q = x.torch.zeros((len(lens), rows, heads, hd), dtype=x.tdt, device=x.e.device)
    q[..., 0] = 2.0 ** (power - power // 2)
    q[:, ::2, :, 0] *= -1
    q[:, :, 1, 0] *= -1
    K, V = x.ref.rows(0)
    for hint in (max(lens), 0):
        out = x.rows(q.shape)
        x.B.dflash_kvq_attention(x.e, x.batch(lens, hint), x.cache, 0, q, out)
        x.e.device_status()
        got, ref = f64(out), km.attention64(f64(q), K, V, x.table, lens, counts, True, x.n_pages)[0]
        n = max(lens) + rows
        # exact scores, so weights that are off by the roundings of exponentials (2^-22 with the exponent's) and, in bf16, of weights, and sums of n; and the output's rounding
        v = np.abs(V[np.isfinite(V)]).max()
        tol = v * (2 * (n + 64) * 2.0 ** -24 + 2.0 ** -22 + (2.0 ** -7 if dtype == "bf16" else 0)) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref)
        assert np.isfinite(got).all() and (np.abs(got - ref) <= tol).all(), (power, hint, float(np.abs(got - ref).max()))


def _pair_bound(ref, slack, wabs, dtype):
    """bf16 weights as hi + lo: hi is off by 2^-8 of itself at most and lo holds that to 2^-8 of it, so weights by 2^-16 and their shares by twice that; the output's rounding, 2^-8 of
    the value."""
    if dtype == "f32":
        return km.allowed(ref, slack, wabs, dtype)
    return slack + 2.0 ** -15 * (1 + 2.0 ** -8) * wabs + 2.0 ** -8 * (1 + 2.0 ** -7) * np.abs(ref)


@pytest.mark.parametrize("heads,kv,hd,bits,rows,lens", [(4, 1, 128, (8, 8), 1, (3, 4, 2, 6, 1)), (8, 2, 64, (4, 8), 6, (2, 0, 9)), (8, 2, 96, (4, 4), 16, (1, 5)), (10, 2, 80, (8, 4), 3, (7, 2, 700)),
                                                        (32, 8, 128, (4, 4), 17, (800, 5))])
def test_bf16_weights_are_held_to_sixteen_bits(heads, kv, hd, bits, rows, lens):
    """Few keys, whose values cancel in some dims: there the output's own rounding is small, and weights of eight bits would be seen."""
    counts = (rows,) * len(lens)
    x = Setup("bf16", heads, kv, hd, bits, len(lens), [n + rows for n in lens], seed=hd + rows, scales=(124, 129))
    x.poison(lens, counts)
    x.upload()
    q, out = x.rows((len(lens), rows, heads, hd), 0.1), x.rows((len(lens), rows, heads, hd))
    x.B.dflash_kvq_attention(x.e, x.batch(lens), x.cache, 1, q, out)
    x.e.device_status()
    ref, slack, wabs = km.attention64(f64(q), *x.ref.rows(1), x.table, lens, counts, True, x.n_pages)
    over = np.abs(f64(out) - ref) / np.maximum(_pair_bound(ref, slack, wabs, "bf16"), 1e-30)
    assert over.max() <= 1, float(over.max())


@pytest.mark.parametrize("dtype,hd,bits,rows", [("bf16", 128, (4, 4), 1), ("bf16", 64, (8, 8), 40), ("f32", 48, (4, 8), 5), ("bf16", 32, (8, 4), 9)])
def test_values_beyond_the_type_are_infinities(dtype, hd, bits, rows):
    """Codes that stand for more than the type's largest number: an infinity of their sign in the rows that see the key, whatever its weight, among keys that all rows see and behind."""
    heads, kv, lens = 4, 2, (200, 2000)
    counts = (rows, rows)
    x = Setup(dtype, heads, kv, hd, bits, 2, [n + rows for n in lens], seed=rows, scales=(120, 124))
    x.poison(lens, counts)
    (at, shift), e_at = x.ref.at[1], x.ref.at[3]
    b = bits[1]
    hits = [(0, 5, 0, 3, 0), (0, 200 + rows - 1, 1, 1, 1), (1, 1203, 0, hd - 1, 1), (1, 40, 1, 0, 0), (1, 2000, 1, 2, 0)]   # sequence, position, head, dim, sign
    for s, p, h, d, neg in hits:
        unit, key = x.ref.data[:, x.table[s, p // PAGE], h], p % PAGE
        blk = d // 32
        unit[:, at[key, blk]] = 0
        sh = int(shift[key, blk, d % 32])
        unit[:, at[key, blk, d % 32]] |= ((6 if b == 4 else 0x78) | ((8 if b == 4 else 0x80) if neg else 0)) << sh      # 4 or 256 ...
        unit[:, e_at[key, blk]] = 253 if b == 4 else 247                                                              # ... times 2^126 or 2^120
    x.upload()
    q, out = x.rows((2, rows, heads, hd), 0.5), x.rows((2, rows, heads, hd))
    before = out.clone()
    want = {}
    for s, p, h, d, neg in hits:
        for j in range(rows):
            if p <= lens[s] + j:
                for g in range(heads // kv):
                    want[(s, j, h * (heads // kv) + g, d)] = -np.inf if neg else np.inf
    x.B.dflash_kvq_attention(x.e, x.batch(lens), x.cache, 0, q, out)
    x.e.device_status()
    got = f64(out)
    bad = ~np.isfinite(got)
    assert {tuple(int(i) for i in at_): got[tuple(at_)] for at_ in np.argwhere(bad)} == want
    # the other elements as if the values were not there
    ref, slack, wabs = km.attention64(f64(q), *(np.where(np.abs(t) > 2.0 ** 127, 0.0, t) for t in x.ref.rows(0)), x.table, lens, counts, True, x.n_pages)
    tol = _pair_bound(ref, slack, wabs, dtype)
    assert (np.abs(got - ref)[~bad] <= tol[~bad]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
def test_every_code_and_scale_is_read_back_rounded_once(dtype, bits):
    """255 pages, one a scale from 2^-127 to 2^127; every code in every place of a row by turns.  Numbers below the smallest normal one keep the bits that the type has for them."""
    x = Setup(dtype, 2, 1, 64, (bits, bits), 1, [255 * PAGE], layers=1, extra=0)
    n = 16 if bits == 4 else 256
    for part in (0, 1):
        at, shift = x.ref.at[part]
        code = (np.arange(255)[:, None, None, None] * 5 + np.arange(PAGE)[:, None, None] * 16 + np.arange(2)[:, None] * 32 + np.arange(32)) % n
        if bits == 8:
            code = np.where(code & 127 == 127, code ^ 1, code)
        data = np.zeros((255, x.ref.data.shape[-1]), np.int64)
        for page in range(255):
            np.add.at(data[page], at.ravel(), (code[page] << shift).ravel())
        used = np.unique(at)
        where = x.table[0, :255]
        x.ref.data[0, where[:, None], 0, used[None, :]] = data[:, used].astype(np.uint8)
        x.ref.data[0, where[:, None], 0, x.ref.at[2 + part].ravel()[None, :]] = np.arange(255)[:, None]
    x.upload()
    rows = 255 * PAGE
    k, v = (x.torch.full((1, rows, 1, 64), 9.0, dtype=x.tdt, device=x.e.device) for _ in range(2))
    x.B.dflash_kvq_read(x.e, x.batch([0], 0), x.cache, 0, k, v, x.ints([0]))
    x.e.device_status()
    for got, want in zip((k, v), x.ref.rows(0)):
        want = x.torch.from_numpy(np.ascontiguousarray(want[x.table[0, :255]].reshape(1, rows, 1, 64))).to(x.tdt)
        same = (got.cpu() == want) | (want == 0) & (got.cpu() == 0)
        bad = (~same).nonzero()
        assert not len(bad), (len(bad), [(int(b[1]) // PAGE, float(got[tuple(b)]), float(want[tuple(b)])) for b in bad[:5]])
