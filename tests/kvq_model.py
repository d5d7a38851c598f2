"""Test side of the caches held in 4 or 8 bits: the format and its layout element by element in numpy, attention in 64 bits, and the error that the kernels' roundings allow."""
import numpy as np

PAGE = 16
LARGEST = {4: 6.0, 8: 448.0}


def blocks(hd):
    return (hd + 31) // 32


def scale_row(nb):
    return 4 if nb == 3 else nb


def unit_bytes(hd, kb, vb):
    return 64 * blocks(hd) * (kb + vb) + 2 * PAGE * scale_row(blocks(hd))


def code_values(bits):
    """Values of the codes with a clear sign bit, 8-bit code 127 (NaN) left out."""
    M, bias = (1, 1) if bits == 4 else (3, 7)
    n = 8 if bits == 4 else 127
    c = np.arange(n)
    m, x = c & ((1 << M) - 1), c >> M
    return np.where(x > 0, (1 + m / 2.0 ** M) * 2.0 ** (x - bias), m / 2.0 ** M * 2.0 ** (1 - bias))


def quantise(x, bits):
    """[..., hd] float64 (any, infinities and NaN too) -> codes [..., NB, 32], e [..., NB]."""
    hd = x.shape[-1]
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (-hd % 32,))], -1).reshape(x.shape[:-1] + (blocks(hd), 32))
    most, limit = np.abs(x).max(-1), 7.0 if bits == 4 else 464.0
    bad = ~np.isfinite(x).all(-1)
    most = np.where(bad, 0.0, most)
    e = np.zeros(most.shape, np.int64)
    for t in range(1, 255):                      # the least e that is enough
        e = np.where(most / 2.0 ** (e - 127) > limit, t, e)
    y = np.where(bad[..., None], 0.0, x) / 2.0 ** (e[..., None] - 127.0)
    v = code_values(bits)
    a = np.abs(y)
    hi = np.clip(np.searchsorted(v, a), 0, len(v) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = v[hi] - a, a - v[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (a >= v[hi]), hi, lo)
    code = code | np.where(np.signbit(y), 8 if bits == 4 else 128, 0)
    return code.astype(np.uint8), np.where(bad, 255, e).astype(np.uint8)


def values(code, e, bits, hd):
    """codes [..., NB, 32], e [..., NB] -> float64 [..., hd]."""
    v = code_values(bits)
    if bits == 8:
        v = np.append(v, np.nan)
    sign = 8 if bits == 4 else 128
    x = np.where(code & sign, -1.0, 1.0) * v[code & (sign - 1)]
    with np.errstate(invalid="ignore"):
        x = x * np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127))[..., None]
    return x.reshape(x.shape[:-2] + (-1,))[..., :hd]


def places(hd, kb, vb):
    """Byte of a page of a head, and shift, for the codes [16, NB, 32] of K and of V, and the bytes [16, NB] of their scales."""
    nb = blocks(hd)
    key, b, d = np.meshgrid(np.arange(PAGE), np.arange(nb), np.arange(32), indexing="ij")
    q, k = key // 4, key % 4
    if kb == 4:
        k_at, k_shift = (b * 16 + key) * 16 + d // 2, d % 2 * 4
    else:
        k_at, k_shift = ((d // 16 * nb + b) * 16 + key) * 16 + d % 16, 0 * d
    v0 = 64 * nb * kb
    if vb == 4:
        v_at, v_shift = ((q * 16 + d % 16) * nb + b) * 4 + k, d // 16 * 4
    else:
        wide = np.minimum(2, nb - b // 2 * 2)
        v_at, v_shift = b // 2 * 1024 + ((q * 16 + d % 16) * wide + b % 2) * 8 + k * 2 + d // 16, 0 * d
    s0 = v0 + 64 * nb * vb
    sc = np.arange(PAGE)[:, None] * scale_row(nb) + np.arange(nb)[None, :]
    return (k_at, k_shift), (v0 + v_at, v_shift), s0 + sc, s0 + PAGE * scale_row(nb) + sc


class Cache:
    """data [layers, pages, heads, unit] as numpy bytes."""

    def __init__(self, data, hd, kb, vb):
        self.data, self.hd, self.bits = data, hd, (kb, vb)
        self.at = places(hd, kb, vb)

    def put(self, layer, page, key, k, v):
        """K and V rows [heads, hd] of one key."""
        for part, x in enumerate((k, v)):
            code, e = quantise(np.asarray(x, np.float64), self.bits[part])
            at, shift = (a[key] for a in self.at[part])
            unit = self.data[layer, page]
            if self.bits[part] == 4:
                for half in (0, 4):
                    here = shift == half
                    unit[:, at[here]] = (unit[:, at[here]] & (0xF0 >> half)) | (code[:, here] << half)
            else:
                unit[:, at] = code
            unit[:, self.at[2 + part][key]] = e

    def rows(self, layer):
        """K and V in float64, [pages, 16, heads, hd]."""
        out = []
        for part in (0, 1):
            at, shift = self.at[part]
            code = self.data[layer][:, :, at] >> shift.astype(np.uint8)
            if self.bits[part] == 4:
                code = code & 15
            out.append(values(code, self.data[layer][:, :, self.at[2 + part]], self.bits[part], self.hd).transpose(0, 2, 1, 3))
        return out


def attention64(q, k, v, table, lens, counts, causal, n_pages):
    """q [S, R, Hq, hd]; k, v [page, key, Hkv, hd], float64.  (outputs, error that fp32 sums may add, averages of |v| with the rows' weights); rows that are not
    there stay NaN in the outputs' place; dims with a NaN among their keys have no error."""
    S, R, Hq, hd = q.shape
    group = Hq // k.shape[2]
    out, slack, wabs = np.full_like(q, np.nan), np.zeros((S, R, Hq, 1)), np.zeros_like(q)
    for s in range(S):
        n = min(int(lens[s]) + int(counts[s]), table.shape[1] * PAGE)
        pos = np.arange(n)
        ids = table[s][pos // PAGE]
        there = (ids >= 0) & (ids < n_pages)
        for j in range(int(counts[s])):
            at = pos[there & (pos <= int(lens[s]) + j if causal else True)]
            for h in range(Hq):
                if not len(at):
                    out[s, j, h] = 0.0
                    continue
                K, V = k[table[s][at // PAGE], at % PAGE, h // group], v[table[s][at // PAGE], at % PAGE, h // group]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = K @ q[s, j, h] / hd ** 0.5
                    p = np.exp(x - x.max())
                    w = p / p.sum()
                    out[s, j, h], wabs[s, j, h] = w @ V, w @ np.abs(V)
                    # hd products and a sum in fp32 for a score, the scale's rounding and that of the exponent's argument; a score off by d moves the row by at most
                    # 2 d max|v|; as many additions as keys, wavefronts and ranges in the two sums
                    score = (hd + 8) * 2.0 ** -24 * (np.abs(K) @ np.abs(q[s, j, h])).max() / hd ** 0.5 + 8 * 2.0 ** -24 * np.abs(x).max()
                    slack[s, j, h] = np.abs(V[:, np.isfinite(V).all(0)]).max(initial=0.0) * (2 * score + 2 * (len(at) + 64) * 2.0 ** -24)
    return out, slack, wabs


def allowed(ref, slack, wabs, dtype):
    """bf16: probabilities p_i (1 + d_i), |d_i| <= 2^-8, divided by their own sum: weights w_i (1 + d_i) / (1 + mean d), off by at most 2 * 2^-8 / (1 - 2^-8) of
    themselves, and the output's rounding, half a step, 2^-8 of the value.  fp32: the division's and the output's roundings."""
    if dtype == "f32":
        return slack + 2.0 ** -22 * np.abs(ref)
    return slack + 2.0 ** -7 / (1 - 2.0 ** -8) * wabs + 2.0 ** -8 * (1 + 2.0 ** -7) * np.abs(ref)
