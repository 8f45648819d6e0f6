"""How the walks of dk and dv of packed documents are cut (csrc/walk_parts.h), as the host's compiler sees it: for every size that the
operator takes, parts of at least one block that cover their walk, no more of them than the workspace has room for."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include <cstdio>
#include "walk_parts.h"
int main() {   // lines of: blocks of all walks, key heads, shares, least, a walk -> its share, parts
  unsigned long long all;
  int heads, units, least, walk;
  while (std::scanf("%llu %d %d %d %d", &all, &heads, &units, &least, &walk) == 5) {
    const int share = dapple::walk_share(all, heads, units, least);
    std::printf("%d %d\\n", share, share > 0 ? dapple::walk_parts(walk, share) : 0);
  }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("walk_parts")
    (at / "cut.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2007_01045_amd", "csrc"), str(at / "cut.cpp"), "-o", str(at / "cut")], check=True)

    def run(lines):
        text = "".join("%d %d %d %d %d\n" % line for line in lines)
        out = subprocess.run([str(at / "cut")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]

    return run


def test_one_document_of_all_sizes(cut):
    # a single document, both directions: every tile's walk is every block of the rows, for each of the sharing heads
    lines = []
    for rows in (1, 31, 64, 5000, 1 << 20, 1 << 24, 27_000_000, 30_000_000, (1 << 26) - 8):
        for tile, block in ((32, 32), (64, 32), (64, 64), (128, 64), (128, 32)):
            for A, Ak in ((1, 1), (3, 1), (2, 2), (28, 7)):
                if -(-rows // 32) * (A + Ak) >= (1 << 23) - 2048:      # (refused)
                    continue
                walk, tiles = -(-rows // block) * (A // Ak), -(-rows // tile)
                for units in (170, 256):
                    for factor in (1, 2):      # (2: causal, half of all pairs; the longest walk is still a whole one)
                        lines.append((max(1, walk * tiles // factor), Ak, units, 16, walk))
    assert len(lines) > 500
    for (total, heads, units, least, walk), (share, parts) in zip(lines, cut(lines)):
        assert share == min(1 << 30, max(least, -(-total * heads // units))), (total, heads, units, walk)
        assert parts == (-(-walk // share) if walk > share else 1) and parts * share >= walk
        assert (parts - 1) * heads <= units, "more tasks than there is room for"


def test_shares_beyond_an_int(cut):
    # fp32, 30 000 000 rows that all see each other: 468 750 walks of 937 500 blocks, a share that 32 bits do not hold
    rows = 30_000_000
    walk = -(-rows // 32)
    for total in (walk * (rows // 64), walk * (rows // 32), 1 << 44, (170 << 31) - 1, 170 << 31, (170 << 32) - 169, (170 << 32) + 1):
        (share, parts), = cut([(total, 1, 170, 16, walk)])
        assert share >= min(-(-total // 170), walk) and share < (1 << 31) - 1 and parts == 1, (total, share, parts)
