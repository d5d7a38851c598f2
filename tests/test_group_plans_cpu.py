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
