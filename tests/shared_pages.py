"""Test side of the sequences that share pages: a ledger kept entry by entry in Python, attention in 64 bits over unpacked pages, and the error that
the kernels' roundings allow."""
from types import SimpleNamespace

import numpy as np
import torch

PAGE = 16


def dims(n_layers, heads, kv_heads, hd, d=64):
    return SimpleNamespace(n_layers=n_layers, d_model=d, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=hd, d_ffn=64, vocab=64, rope_theta=1e4,
                           rms_eps=1e-6, qk_norm=False, n_experts=0, top_k=0, d_expert=0)


def unpack(pool, layer, heads, hd):
    """(K, V) of one layer, [page, key, head, dim], from the pool's page layout ([layer, page, head, K|V, 16 * hd], any type)."""
    x = pool[layer]
    k = x[:, :, 0].reshape(-1, heads, hd // 8, PAGE, 8).permute(0, 3, 1, 2, 4).reshape(-1, PAGE, heads, hd)
    v = x[:, :, 1].reshape(-1, heads, hd // 16, 4, 16, 4).permute(0, 3, 5, 1, 2, 4).reshape(-1, PAGE, heads, hd)
    return k, v


def attention64(q, k, v, table, lens, causal, n_pages):
    """q [S, R, Hq, hd]; k, v [page, key, Hkv, hd], all float64 on the CPU.  (outputs, error that the kernels' fp32 sums may add per row of bf16 or fp32
    inputs, averages of |v| with the rows' weights).  Keys on entries outside the pool are not there; a row without keys is zeros."""
    S, R, Hq, hd = q.shape
    Hkv = k.shape[2]
    out, slack, wabs = torch.zeros_like(q), torch.zeros(S, R, Hq, 1, dtype=torch.float64), torch.zeros_like(q)
    for s in range(S):
        n = min(int(lens[s]) + R, table.shape[1] * PAGE)
        pos = np.arange(n)
        ids = table[s][pos // PAGE]
        there = (ids >= 0) & (ids < n_pages)
        for j in range(R):
            see = there & (pos <= int(lens[s]) + j if causal else True)
            at = pos[see]
            if not len(at):
                continue
            for h in range(Hq):
                K, V = k[ids[see], at % PAGE, h * Hkv // Hq], v[ids[see], at % PAGE, h * Hkv // Hq]
                x = K @ q[s, j, h] / hd ** 0.5
                out[s, j, h] = torch.softmax(x, 0) @ V
                wabs[s, j, h] = torch.softmax(x, 0) @ V.abs()
                # hd products and a sum in fp32 for a score, the scale's rounding and that of the exponent's argument; a score off by d moves the row by at
                # most 2 d max|v|; as many additions as keys and parts in the two sums
                score = (hd + 8) * 2.0 ** -24 * float((K.abs() @ q[s, j, h].abs()).max() / hd ** 0.5 + x.abs().max())
                slack[s, j, h] = float(V.abs().max()) * (2 * score + 2 * (len(at) + 64) * 2.0 ** -24)
    return out, slack, wabs


def allowed(ref, slack, wabs, dtype):
    """bf16: the output's rounding, and that of the probabilities as a hi + lo pair of bf16 numbers: hi is off by at most 2^-8 of the value, lo by 2^-8 of that, 2^-16 of
    every weight w_i, so the row by at most 2^-16 sum w_i |v_i| = 2^-16 wabs."""
    if dtype == "f32":
        return slack + 2.0 ** -23 * ref.abs()
    return slack + 2.0 ** -16 * wabs + 2.0 ** -8 * ref.abs()


class LedgerModel:
    """What the dflash_pages_* calls do, entry by entry."""

    def __init__(self, rows, width, n_pages):
        self.table = np.full((rows, width), -1, np.int32)
        self.lens = np.zeros(rows, np.int32)
        self.anchor = np.zeros(rows, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.copies = []        # (from, to, rows) of the last call

    def _ok(self, i):
        return 0 <= i < len(self.refs)

    def _drop(self, r, p):
        if self._ok(self.table[r, p]):
            self.refs[self.table[r, p]] -= 1
        self.table[r, p] = -1

    def fork(self, parents, children):
        self.copies = []
        for a, b in zip(parents, children):
            for p in range(self.table.shape[1]):
                self._drop(b, p)
            for p in range(min(-(-int(self.lens[a]) // PAGE), self.table.shape[1])):
                self.table[b, p] = self.table[a, p]
                if self._ok(self.table[b, p]):
                    self.refs[self.table[b, p]] += 1
            self.lens[b], self.anchor[b] = self.lens[a], self.anchor[a]

    def release(self, rows, keep=None):
        self.copies = []
        for i, r in enumerate(rows):
            k = 0 if keep is None else keep[i]
            for p in range(-(-k // PAGE), self.table.shape[1]):
                self._drop(r, p)
            self.lens[r] = min(self.lens[r], k)

    def reserve(self, tokens):
        self.copies = []
        free = [i for i in range(len(self.refs)) if self.refs[i] == 0]
        before, asked, stuck, state = self.refs.copy(), {}, False, []
        takes = []
        for r, t in enumerate(tokens):
            n = int(self.lens[r])
            span = range(n // PAGE, -(-(n + int(t)) // PAGE)) if t > 0 else range(0)
            if t > 0 and span.stop > self.table.shape[1]:
                state.append(None)
                continue
            state.append(span)
            want = []
            for p in span:
                i = int(self.table[r, p])
                if not self._ok(i):
                    want.append(p)
                elif p == span.start:
                    if asked.get(i, 0) < before[i] - 1:
                        want.append(p)
                    asked[i] = asked.get(i, 0) + 1
                elif before[i] > 1:
                    want.append(p)
            takes.append((r, want, n))
        used = 0
        for r, want, n in takes:
            used += len(want)
            stuck = stuck or used > len(free)
            if stuck:
                continue
            for p in want:
                old, new = int(self.table[r, p]), free[used - len(want) + want.index(p)]
                self.table[r, p] = new
                self.refs[new] += 1
                if self._ok(old):
                    self.refs[old] -= 1
                    if p == n // PAGE and n % PAGE:
                        self.copies.append((old, new, -(-(n % PAGE) // 4) * 4))
        return np.array([0 if sp is None else int(all(self._ok(self.table[r, p]) and self.refs[self.table[r, p]] == 1 for p in sp))
                         for r, sp in enumerate(state)], np.int32)

    def compact(self):
        alive = np.flatnonzero(self.refs > 0)
        n = len(alive)
        holes = [i for i in range(n) if self.refs[i] <= 0]
        self.copies = []
        table = self.table.copy()
        for a, b in zip([int(i) for i in alive if i >= n], holes):
            self.copies.append((a, b, PAGE))
            table[self.table == a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = table
        return n

    def apply_copies(self, pool, hd):
        """The call's copies in a pool [layer, page, head, K|V, 16 * hd] on the CPU."""
        at = torch.arange(PAGE * hd)
        for part, key in ((0, at // 8 % PAGE), (1, at // 64 % 4 * 4 + at % 4)):
            for a, b, rows in self.copies:
                here = torch.nonzero(key < rows)[:, 0]
                pool[:, b, :, part, here] = pool[:, a, :, part, here]
