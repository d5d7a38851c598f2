"""The 4- and 8-bit format of the test side against its definition, and the sizes and refusals that need no GPU."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from tests import kvq_model as km


def test_codes_round_to_the_nearest_value():
    rng = np.random.RandomState(0)
    for bits in (4, 8):
        x = rng.standard_normal((64, 96)) * 2.0 ** rng.randint(-30, 30, (64, 1))
        x[3] = 0
        code, e = km.quantise(x, bits)
        y = km.values(code, e, bits, 96)
        blocks = np.abs(x).reshape(64, 3, 32).max(-1)
        scale = 2.0 ** (e.astype(float) - 127)
        limit = km.LARGEST[bits] + (1 if bits == 4 else 16)
        assert (blocks <= limit * scale).all() and ((blocks > limit * scale / 2) | (blocks == 0)).all()
        # no code is nearer
        all_values = np.concatenate([-km.code_values(bits), km.code_values(bits)])
        nearest = np.abs((x.reshape(64, 3, 32) / scale[..., None])[..., None] - all_values).min(-1)
        assert np.allclose(np.abs(x - y).reshape(64, 3, 32), nearest * scale[..., None], rtol=1e-12, atol=0)


def test_ties_go_to_even_codes():
    x = np.zeros(32)
    x[:9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    code, e = km.quantise(x, 4)
    assert e[0] == 127 and list(code[0, :9]) == [7, 0, 2, 2, 4, 4, 6, 6, 14]


def test_blocks_that_are_not_finite():
    x = np.ones((3, 64))
    x[0, 5], x[1, 40], x[2, 33] = np.nan, np.inf, -np.inf
    for bits in (4, 8):
        code, e = km.quantise(x, bits)
        assert [list(r == 255) for r in e] == [[True, False], [False, True], [False, True]]
        y = km.values(code, e, bits, 64)
        assert np.isnan(y[0, :32]).all() and np.isfinite(y[0, 32:]).all() and np.isnan(y[1, 32:]).all()


@pytest.mark.parametrize("hd", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("kb,vb", [(4, 4), (8, 8), (8, 4), (4, 8)])
def test_layout_uses_every_place_once(hd, kb, vb):
    (k, ks), (v, vs), k_sc, v_sc = km.places(hd, kb, vb)
    bits = np.concatenate([(k * 8 + ks).ravel(), (v * 8 + vs).ravel()])
    assert len(np.unique(bits)) == len(bits) and bits.max() < 8 * k_sc.min()
    scales = np.concatenate([k_sc.ravel(), v_sc.ravel()])
    assert len(np.unique(scales)) == len(scales) and scales.max() < km.unit_bytes(hd, kb, vb)


def _dims(B, **kw):
    d = dict(n_layers=3, d_model=64, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ffn=64, vocab=64, rope_theta=1e4, rms_eps=1e-6, qk_norm=0, dtype=B.DFLASH_BF16,
             n_experts=0, top_k=0, d_expert=0)
    d.update(kw)
    return B.Dims(*[d[n] for n, _ in B.Dims._fields_])


def test_sizes():
    from paper_2602_06036_amd import binding as B
    l = B.lib()
    for hd in (16, 48, 64, 80, 96, 128):
        for kb in (4, 8):
            for vb in (4, 8):
                d = _dims(B, head_dim=hd, n_q_heads=4)
                assert l.dflash_kvq_bytes(C.byref(d), 7, kb, vb) == 3 * 7 * 2 * km.unit_bytes(hd, kb, vb)
    # past 32 bits
    d = _dims(B, n_layers=36, n_kv_heads=8, n_q_heads=32, head_dim=128, d_model=4096)
    assert l.dflash_kvq_bytes(C.byref(d), 1 << 20, 4, 4) == 36 * (1 << 20) * 8 * 2176


def test_refusals_without_a_context():
    from paper_2602_06036_amd import binding as B
    l = B.lib()
    for n, kb, vb, word in ((0, 4, 4, b"n_pages"), (-3, 4, 4, b"n_pages"), (5, 3, 4, b"bits"), (5, 4, 16, b"bits"), (5, 0, 8, b"bits")):
        assert l.dflash_kvq_bytes(C.byref(_dims(B)), n, kb, vb) == 0 and word in l.dflash_last_error(None)
    assert l.dflash_kvq_bytes(None, 5, 4, 4) == 0
    assert l.dflash_kvq_bytes(C.byref(_dims(B, head_dim=72)), 5, 4, 4) == 0 and b"head_dim" in l.dflash_last_error(None)
    b, q = B.Batch(), B.Kvq()
    assert l.dflash_kvq_write(None, C.byref(b), C.byref(q), 0, 1, None, None, None, None) == B.DFLASH_EINVAL
    assert l.dflash_kvq_read(None, C.byref(b), C.byref(q), 0, 1, None, None, None, None, None) == B.DFLASH_EINVAL
    assert l.dflash_kvq_attention(None, C.byref(b), C.byref(q), 0, 1, None, 1, None, None, None) == B.DFLASH_EINVAL
    assert l.dflash_kvq_pack(None, C.byref(b), C.byref(q), None, None) == B.DFLASH_EINVAL
    assert l.dflash_kvq_unpack(None, C.byref(b), C.byref(q), None, None) == B.DFLASH_EINVAL


# ---- launch rules, compiled for the host, and the waits of the sweep ----------------------------------------------------------
CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2602_06036_amd", "csrc")
DRIVER = r"""
#include <stdio.h>
#include "plan.h"
int main() {
  int seqs, rows, hq, hkv, bf16, wide, tokens;
  long long part_rows;
  float all;
  while (scanf("%d %d %d %d %d %d %d %lld %f", &seqs, &rows, &hq, &hkv, &bf16, &wide, &tokens, &part_rows, &all) == 9) {
    const KvqPlan p = kvq_plan(seqs, rows, hq, hkv, bf16 != 0, wide != 0, tokens, part_rows);
    printf("%d %d %d\n", p.tiles, p.parts, p.parts ? kvq_chunk(all, p.parts) : 0);
  }
}
"""


def test_ranges_fit_their_places_whatever_the_lengths(tmp_path):
    (tmp_path / "p.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    rng = np.random.RandomState(0)
    queries, lens = [], []
    for seqs in (1, 2, 3, 7, 16, 48, 64, 65, 150, 1000, 2000):
        for rows in (1, 2, 16, 17, 400):
            for hq, hkv in ((32, 8), (4, 4), (10, 2), (16, 1)):
                for part_rows in (98304, seqs * rows * hq, 64 * rows * hq, 3 * rows * hq - 1):
                    n = rng.randint(0, int(rng.choice([40, 4000, 300000])), seqs)
                    n[rng.randint(seqs)] = rng.choice([0, 1, 9000, 2 ** 28])
                    pairs = -(-n // 32)
                    all_fours = np.float32(0)
                    for s0 in range(0, seqs, 64):       # as the device adds them up
                        all_fours = np.float32(all_fours + np.float32((-(-pairs[s0:s0 + 64] // 4)).sum()))
                    # a hint that has little to do with the lengths
                    queries.append((seqs, rows, hq, hkv, rng.randint(2), rng.randint(2), int(rng.choice([1, 256, 257, 5000, 40000])), part_rows, repr(float(all_fours))))
                    lens.append(n)
    out = subprocess.run([str(tmp_path / "p")], input="\n".join(" ".join(str(x) for x in q) for q in queries), capture_output=True, text=True, check=True).stdout
    cut = 0
    for (seqs, rows, hq, hkv, bf16, wide, tokens, part_rows, _), n, line in zip(queries, lens, out.splitlines()):
        tiles, parts, chunk = (int(x) for x in line.split())
        tile = 16 if not bf16 or rows * hq // hkv <= 16 else 32 if rows * hq // hkv <= 32 or not wide else 64
        assert tiles == -(-rows * hq // hkv // tile)
        if parts:
            cut += 1
            assert chunk % 128 == 0 and chunk >= 256
            assert (parts + seqs) * rows * hq <= part_rows
            assert int((-(-n // chunk)).sum()) <= parts + seqs, (seqs, parts, chunk)
    assert cut > 100 and cut < len(queries)


@pytest.mark.skipif(not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")), reason="needs hipcc")
def test_the_sweep_waits_for_its_pair_and_not_for_the_next(tmp_path):
    """A turn waits until its own pair's copies have landed, the next pair's (two pages of three copies) in flight.  The compiler does not see the copies: whatever load it
    waits for by itself drains them all, so such a wait may stand only where page ids are loaded or taken over, and behind the last pair."""
    from paper_2602_06036_amd import build
    with open(os.path.join(CSRC, "kvq_attn.hip")) as f:
        kernels = f.read().split("template <typename T, int NB, int KB, int VB>\nvoid launch(")[0]      # without what makes all others of them
    (tmp_path / "k.hip").write_text(kernels + "".join("template __global__ void kvq_attn_kernel<bf16_t, 4, 4, 4, %d>(KvqAttn);\n" % rb for rb in (1, 2, 4)) + "}\n")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--offload-device-only", "-S", "-I", CSRC, str(tmp_path / "k.hip"), "-o", str(tmp_path / "k.s")],
                   check=True, capture_output=True)
    asm = (tmp_path / "k.s").read_text()
    for rb in (1, 2, 4):
        body = re.search(r"^_ZN\S*kvq_attn_kernelItLi4ELi4ELi4ELi%dEEEv7KvqAttn:.*?^\.Lfunc_end" % rb, asm, re.S | re.M).group(0)
        loops = {}
        for b in re.split(r"^(?=\.LBB\d+_\d+:|; %bb\.\d+:)", body, flags=re.M):
            m = re.search(r"Header=(BB\d+_\d+) ", b) or re.match(r"\.L(BB\d+_\d+):.*Loop Header", b)
            if m:
                loops.setdefault(m.group(1), []).append(b)
        sweep = [bs for bs in loops.values() if any("global_load_lds" in b for b in bs) and any("mfma" in b for b in bs)]
        assert len(sweep) == 1, rb
        waits = [(int(n), "global_load_lds" in b, "mfma" in b or "ds_read" in b) for b in sweep[0] for n in re.findall(r"s_waitcnt[^\n]*vmcnt\((\d+)\)", b)]
        assert (6, True, False) in waits, (rb, waits)
        assert all(w == (6, True, False) or w == (0, False, False) for w in waits) and len(waits) <= 4, (rb, waits)
