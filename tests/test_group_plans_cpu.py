"""Key ranges of the attention of sequences that share pages (csrc/plan.h), compiled for the host: whatever lengths a call expects, its ranges fit the partial rows
that the workspace holds for its query rows."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2602_06036_amd", "csrc")

DRIVER = r"""
#include <stdio.h>
#include "plan.h"
int main() {
  int tiles, seqs, rows, heads, prefix, own, all, mfma;
  while (scanf("%d %d %d %d %d %d %d %d", &tiles, &seqs, &rows, &heads, &prefix, &own, &all, &mfma) == 8) {
    const GroupSplits g = group_plan(tiles, seqs, rows, heads, prefix, own, all, mfma != 0);
    printf("%d %d %d\n", g.prefix, g.own, group_parts(all));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    (d / "p.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def run(queries):
        out = subprocess.run([str(d / "p")], input="\n".join(" ".join(str(x) for x in q) for q in queries), capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]

    return run


def test_ranges_fit_the_workspace_whatever_the_lengths(plans):
    q = []
    for seqs in (1, 2, 3, 5, 8, 16, 31, 32, 64, 200):
        for block in (1, 2, 7, 16):
            for group, heads in ((1, 4), (4, 8), (8, 4), (64, 1)):
                rows = block * group
                for tile in (64, 128):
                    for extra in (0, seqs - 1):
                        for prefix in (0, 16, 100, 1029, 8192, 16384, 131072):
                            for own in (1, 40, 613, 1531, 16384):
                                q.append((-(-seqs * rows // tile) + extra, seqs, rows, heads, prefix, own, seqs * rows * heads, int(tile == 128)))
    for x, (np, ns, most) in zip(q, plans(q)):
        assert np >= 1 and ns >= 1 and np <= 32 and ns <= 32 and np + ns <= most <= 64, (x, np, ns, most)
        assert np == 1 or np * 4 * 32 <= x[4] + 31 * np, (x, np)          # four pairs of pages a range
    # 32 blocks of 16 rows behind 16384 shared tokens: more ranges than lengths that fill the block table give
    a, b = plans([(16, 32, 64, 8, 16384, 1531, 16384, 1), (16, 32, 64, 8, 17936, 17936, 16384, 1)])
    assert a[0] + a[1] <= a[2] and b[0] + b[1] <= b[2] and a[2] == b[2]


RULES = r"""
#include <stdio.h>
#include "plan.h"
int main() {
  int bf16, heads, kv, hd, seqs, block, prefix, own, knob;
  while (scanf("%d %d %d %d %d %d %d %d %d", &bf16, &heads, &kv, &hd, &seqs, &block, &prefix, &own, &knob) == 9) {
    const int rows = block * (heads / kv), tokens = prefix + own + block;
    const bool mfma = bf16 && hd % 32 == 0;
    const int tile = mfma && seqs * rows > 64 ? 128 : 64;
    const GroupSplits g = group_plan(seqs * rows / tile, seqs, rows, kv, prefix, own + block, seqs * rows * kv, mfma);
    const int blocks = (rows + 63) / 64 * kv;
    const SplitPlan p = plan_splits(seqs, hd == 64 || hd == 128 ? blocks : kv, tokens, 256);
    printf("%d %d %d\n", group_apart(g.us, seqs, rows, kv, tokens, mfma, knob), step_apart(g.us, seqs, blocks, p, knob),
           step_apart_simple(g.us, seqs, rows, kv, hd, tokens, bf16 != 0, p, knob));
  }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(RULES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "r.cpp"), "-o", str(d / "r")], check=True)

    def run(which, queries):
        out = subprocess.run([str(d / "r")], input="\n".join(" ".join(str(x) for x in q) for q in queries), capture_output=True, text=True, check=True).stdout
        return [bool(int(line.split()[which])) for line in out.splitlines()]

    return run


# (bf16, query heads, kv heads, head dim, sequences, rows a sequence, shared tokens, own tokens): microseconds without the groups, with them
STEP_SIMPLE = {   # verification of four layers
    (0, 4, 1, 64, 8, 4, 160, 28): (91, 142), (0, 4, 1, 128, 14, 5, 176, 26): (137, 206), (0, 4, 1, 64, 3, 8, 416, 87): (102, 141), (0, 8, 8, 128, 5, 4, 224, 37): (124, 168),
    (0, 8, 2, 96, 8, 5, 96, 26): (112, 146), (0, 8, 2, 64, 2, 8, 1024, 100): (127, 136), (0, 8, 2, 64, 32, 16, 1024, 200): (820, 362), (0, 8, 2, 64, 8, 4, 2000, 100): (184, 151),
    (0, 16, 2, 96, 36, 8, 5168, 59): (4154, 684), (1, 8, 2, 96, 4, 8, 128, 60): (134, 148), (1, 8, 2, 96, 4, 16, 512, 100): (223, 170), (1, 32, 8, 96, 26, 16, 128, 153): (1169, 262),
    (1, 8, 8, 32, 34, 8, 1520, 219): (965, 181), (1, 32, 8, 112, 17, 8, 416, 388): (1253, 219), (1, 16, 2, 80, 10, 5, 6912, 213): (1289, 218), (1, 8, 2, 32, 8, 4, 2000, 100): (210, 133)}
STEP_MFMA = {     # likewise, 8B and head dim 64
    (1, 32, 8, 128, 32, 16, 16384, 800): (1008, 878), (1, 32, 8, 128, 16, 16, 2048, 600): (290, 304), (1, 32, 8, 128, 32, 4, 8192, 300): (553, 318),
    (1, 32, 8, 128, 8, 8, 8192, 300): (274, 241), (1, 32, 8, 128, 16, 2, 4096, 100): (245, 185), (1, 16, 4, 64, 32, 4, 8192, 300): (522, 209)}
ALONE = {         # dflash_group_attention's launches in such a step
    (1, 8, 2, 96, 4, 8, 128, 60): (140, 148), (1, 8, 2, 96, 2, 8, 1024, 100): (170, 135), (1, 8, 2, 32, 4, 8, 128, 60): (123, 136), (1, 8, 2, 96, 32, 16, 1024, 200): (249, 218),
    (0, 8, 2, 64, 4, 8, 128, 60): (123, 137), (0, 8, 2, 64, 2, 8, 1024, 100): (246, 136), (0, 8, 2, 64, 32, 4, 4096, 200): (424, 227), (1, 8, 2, 80, 4, 16, 512, 100): (229, 165)}


@pytest.mark.parametrize("which,measured", [(0, ALONE), (1, STEP_MFMA), (2, STEP_SIMPLE)], ids=["by_itself", "step_mfma", "step_plain_kernel"])
def test_each_rule_compares_what_it_launches(rules, which, measured):
    """Whether a batch goes sequence by sequence: the faster side of measured ones, except where they are within 10 %; and what the knob says."""
    told = [(q, without, with_groups) for q, (without, with_groups) in measured.items() if max(without, with_groups) > 1.1 * min(without, with_groups)]
    assert len(told) >= 4
    for (q, without, with_groups), apart in zip(told, rules(which, [q + (0,) for q, _, _ in told])):
        assert apart == (without < with_groups), (q, without, with_groups)
    assert all(rules(which, [q + (1,) for q in measured])) and not any(rules(which, [q + (2,) for q in measured]))
