"""Sequences that share pages in the step: that the step attends by the groups where it should, what it gives then, and its capture into a graph.  (The calls by themselves:
test_gpu_shared_pages.py.)"""
from dataclasses import replace

import numpy as np
import pytest

from synth import inputs as si
from tests.helpers import tiny_workload
from tests.test_gpu_graph import _enqueue_step, _outputs, _restore, _snapshot
from tests.test_gpu_shared_pages import ONCE, PAGE, Pair, _shared_model, _torch, dims

pytestmark = pytest.mark.gpu

ATTN = 3          # DFLASH_PROF_ATTN


def _bytes(m, esize, tokens, launches):
    return launches * tokens * 2.0 * m.n_kv_heads * m.head_dim * esize


def _compare_step(w, prompts, children, bound):
    """One step of the forked batch without the groups, with them, and without again.  With them every attention launch of draft and verification reads what is shared
    once (its bytes say so), and the rows are those of the step without within twice the distance `bound` that either may have from exact arithmetic."""
    torch = _torch()
    import paper_2602_06036_amd as dfl
    wt, wd = si.make_weights(w, 8)
    g, led, groups, owner = _shared_model(w, wt, wd, prompts, children, 3)
    S, B = g.S, w.block_size
    dfl.dflash_pages_reserve(g.e, led, torch.full((S,), B, dtype=torch.int32, device=g.dev))
    snap = _snapshot(g)
    prop = np.random.RandomState(3).randint(0, w.target.vocab - 1, size=(S, B - 1))   # the same rows whatever the draft says
    longest, launches, esize = int(g.host_lens.max()), w.target.n_layers + w.draft.n_layers, 2 if w.dtype == "bf16" else 4
    shared = min(groups.prefix_len, longest)
    tokens = {False: S * (longest + B), True: len(prompts) * shared + S * (longest - shared + B)}
    assert tokens[True] < tokens[False]
    outs = []
    for on in (False, True, False):
        _restore(g, snap)
        dfl.dflash_set_groups(g.e, groups if on else None)
        g.e.profile_enable(True)
        g.e.profile_read()
        outs.append(g.step(proposals=prop))
        _, n, read = g.e.profile_read()[ATTN]
        g.e.profile_enable(False)
        assert n == launches and read == _bytes(w.target, esize, tokens[on], launches), (on, n, read)
    plain, once, again = outs
    for k in ("logits_d", "logits_t"):
        assert np.array_equal(plain[k], again[k])                            # switched off: what it was
        assert float(np.abs(plain[k] - once[k]).max()) <= 2 * bound, k
        assert not np.array_equal(plain[k], once[k]), k                      # another order of sums: it did run
    first = {i: owner.index(i) for i in owner}
    for s in range(S):                                                       # samples of one prompt: the same draft
        assert float(np.abs(once["logits_d"][s] - once["logits_d"][first[owner[s]]]).max()) <= 2 * bound
    g.e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd,block", [("f32", 4, 4, 64, 8), ("f32", 6, 2, 48, 5), ("bf16", 8, 2, 128, 16), ("bf16", 8, 2, 64, 8), ("bf16", 4, 2, 96, 8), ("bf16", 4, 2, 80, 3),
                                                        ("bf16", 8, 1, 128, 16), ("bf16", 16, 2, 64, 16)])
def test_step_attends_by_the_groups(dtype, heads, kv, hd, block, monkeypatch):
    """However small the batch, with the plan forced: every kernel of the groups, its rows as the operand of the O projection."""
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    w = tiny_workload(seed=5, n_layers=2, draft_layers=1, vocab=512, block=block, n_seqs=7, ctx=(150, 150), taps=(0,), dtype=dtype, heads=heads, kv_heads=kv, hd=hd)
    prompts = [p[:n] for p, n in zip(si.make_prompts(w), (149, 77))]
    _compare_step(w, prompts, (4, 1), 1e-4 if dtype == "f32" else 2e-2)


def test_step_of_fewer_rows_under_groups(monkeypatch):
    """Groups set once, blocks of 16, 5, 2 and 16 rows chosen per step: every step within the model's distance of the same step without groups."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    import paper_2602_06036_amd as dfl
    w = tiny_workload(seed=9, n_layers=2, draft_layers=1, vocab=512, block=16, n_seqs=5, ctx=(150, 150), taps=(0,), dtype="bf16", heads=8, kv_heads=2, hd=128)
    wt, wd = si.make_weights(w, 8)
    g, led, groups, _ = _shared_model(w, wt, wd, [p[:n] for p, n in zip(si.make_prompts(w), (149, 77))], (2, 1), 4)
    for block in (16, 5, 2, 16):
        dfl.dflash_pages_reserve(g.e, led, torch.full((5,), block, dtype=torch.int32, device=g.dev))
        snap = _snapshot(g)
        prop = np.random.RandomState(block).randint(0, w.target.vocab - 1, size=(5, block - 1))
        outs = []
        for on in (True, False):
            _restore(g, snap)
            dfl.dflash_set_groups(g.e, groups if on else None)
            outs.append(g.step(proposals=prop, block=block))
        for k in ("logits_d", "logits_t"):
            assert float(np.abs(outs[0][k] - outs[1][k]).max()) <= 4e-2 and not np.array_equal(outs[0][k], outs[1][k]), (block, k)
    g.e.close()


@pytest.mark.parametrize("dtype,heads,kv,hd,block,seqs,tokens", [("bf16", 8, 2, 128, 2, 40, 3000), ("bf16", 8, 2, 64, 2, 40, 3000), ("f32", 4, 4, 64, 4, 12, 1100), ("bf16", 8, 2, 96, 4, 9, 600)])
def test_step_takes_the_groups_by_itself(dtype, heads, kv, hd, block, seqs, tokens, monkeypatch):
    """Few rows a sequence behind a long prompt: the estimates choose the groups, in the draft as in the verification."""
    monkeypatch.setenv("DFLASH_GROUP_APART", "0")
    w = tiny_workload(seed=6, n_layers=2, draft_layers=1, vocab=512, block=block, n_seqs=seqs, ctx=(tokens, tokens), taps=(0,), dtype=dtype, heads=heads, kv_heads=kv, hd=hd)
    _compare_step(w, si.make_prompts(w)[:1], (seqs - 1,), 1e-4 if dtype == "f32" else 2e-2)


@pytest.mark.parametrize("dtype,hd,temperature", [("f32", 64, 0.0), ("bf16", 128, 0.0), ("bf16", 128, 0.8), ("bf16", 80, 0.0)])
def test_step_under_groups_in_a_graph(dtype, hd, temperature, monkeypatch):
    """The whole step captured while groups are set, and replayed step after step with eager work between: the same as eagerly, bit for bit."""
    torch = _torch()
    monkeypatch.setenv("DFLASH_GROUP_APART", ONCE)
    import paper_2602_06036_amd as dfl
    steps, S = 4, 7
    w = tiny_workload(seed=8, n_layers=2, draft_layers=1, vocab=512, block=4, n_seqs=S, ctx=(150, 150), taps=(0,), dtype=dtype, heads=8, kv_heads=2, hd=hd)
    wt, wd = si.make_weights(w, 8)
    prompts = [p[:n] for p, n in zip(si.make_prompts(w), (149, 77))]
    g, led, groups, _ = _shared_model(w, wt, wd, prompts, (4, 1), steps + 2)
    dfl.dflash_pages_reserve(g.e, led, torch.full((S,), (steps + 1) * w.block_size, dtype=torch.int32, device=g.dev))
    dfl.dflash_set_groups(g.e, groups)
    rng = torch.tensor([77], dtype=torch.int64, device=g.dev) if temperature else None
    uniforms = torch.from_numpy(si.make_uniforms(replace(w, temperature=temperature), 0).astype(np.float32)).to(g.dev) if temperature else None
    batch = g.e.batch(g.seq_lens, g.block_table, g.anchor, int(g.host_lens.max()) + steps * w.block_size)
    snap = _snapshot(g)

    def step():
        _enqueue_step(g, batch, temperature, rng, uniforms)

    eager = []
    for _ in range(steps):
        step()
        eager.append(_outputs(g))
    g.e.device_status()
    _restore(g, snap)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    for i in range(steps):
        graph.replay()
        got = _outputs(g)
        for k, v in eager[i].items():
            assert np.array_equal(got[k], v), (i, k)
        g.host_lens = got["lens"].astype(np.int64)
        g.read_kv(0, 0, 0, 0, int(got["lens"][0]))
    g.e.device_status()
    assert (eager[-1]["lens"] > snap["lens"].cpu().numpy()).all()
    g.e.close()


def test_reserve_in_a_large_pool():
    """A pool of 100 000 pages: asking for more entries than a workgroup has threads, free pages behind 90 000 that are in use, and in holes between them."""
    torch = _torch()
    p = Pair(torch, "bf16", dims(1, 2, 1, 16), dims(1, 2, 1, 16), 66, 1600, 100_000, 64)
    assert p.reserve([1500 * PAGE] * 60 + [0] * 4).all()
    assert (p.m.refs[:90_000] == 1).all() and not p.m.refs[90_000:].any()
    p.set_lens([1500 * PAGE - 3 - i % 5 for i in range(60)])
    p.fork([0, 0, 59, 59], [61, 64, 62, 65])
    assert p.reserve([20] * 63 + [700]).all()                       # behind everything in use; copies of two tails
    p.release([3, 40], [17, 16 * 700])
    p.release([58])
    assert p.reserve([0] * 58 + [9000 * 2, 0, 40, 3, 3, 5]).all()   # in the holes
    assert list(p.reserve([1] * 40 + [16 * 900] * 24)).count(1) > 40
    p.release([62, 61])
    p.compact()
    p.e.close()
