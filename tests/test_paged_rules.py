"""How paged attention deals its work out (csrc/paged_rules.h), compiled for the host."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HDR = os.path.join(ROOT, "paper_2607_22696_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "paged_rules.h"
int main() {
  long tokens;
  int group, heads, batch, most;
  while (scanf("%ld %d %d %d %d", &tokens, &group, &heads, &batch, &most) == 5) {
    const dsa3d::PagedPlan p = dsa3d::paged_plan(tokens, group, heads, batch, most);
    printf("%d %d %d\n", p.tile, p.splits, p.part);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_rules")
    src, exe = d / "r.cpp", d / "r"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", HDR, str(src), "-o", str(exe)])

    def ask(cases):
        """(tile, splits, part) of each (tokens, group, key heads, requests, most keys)."""
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.check_output([str(exe)], input=text, text=True)
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_parts_are_whole_tiles_and_hold_all_keys(plans):
    r = random.Random(1)
    cases = [(150, 4, 2, 2, 4001), (1, 4, 8, 1, 0), (0, 4, 8, 3, 900), (1616, 4, 8, 6, 16000)]
    cases += [(r.randint(0, 6000), r.choice((1, 2, 3, 4, 16)), r.choice((1, 2, 6, 8, 24)),
               r.randint(1, 100), int(2 ** r.uniform(0, 18))) for _ in range(2000)]
    for case, (tile, splits, part) in zip(cases, plans(cases)):
        assert tile in (32, 128) and 1 <= splits <= 64, case
        assert part % 128 == 0, (case, part)  # 128 keys, or 64 or 32, per tile


def test_workloads(plans):
    """Single tokens of 64 requests, of one; chunks beside single tokens; one chunk."""
    assert plans([(64, 4, 8, 64, 8000), (1, 4, 8, 1, 700), (1616, 4, 8, 6, 16000),
                  (1024, 4, 8, 1, 16384)]) == \
        [(32, 4, 1024), (32, 1, 512), (128, 3, 4096), (128, 4, 4096)]
