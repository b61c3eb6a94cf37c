"""How attention over an 8- or 4-bit cache deals its work out: the host's plan (csrc/paged_rules.h,
compiled here) and the division that the kernels make of it by the lengths, written out in numpy."""
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HDR = os.path.join(ROOT, "paper_2607_22696_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "paged_rules.h"
int main() {
  long tokens;
  int group, heads, batch, most, dim;
  while (scanf("%ld %d %d %d %d %d", &tokens, &group, &heads, &batch, &most, &dim) == 6) {
    const dsa3d::MxPlan p = dsa3d::paged_mx_plan(tokens, group, heads, batch, most, dim);
    const int other = dsa3d::paged_plan(tokens, group, heads, batch, most).splits;
    printf("%d %d %d %d %ld %d\n", p.tile, p.splits, p.part, p.target, (long)p.bound, other);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_mx_rules")
    src, exe = d / "r.cpp", d / "r"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", HDR, str(src), "-o", str(exe)])

    def ask(cases):
        """(tile, splits, part, target, bound, paged_plan's splits) of each (tokens, group, key
        heads, requests, most keys, head_dim)."""
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.check_output([str(exe)], input=text, text=True)
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def parts_of(keys, tiles, plan):
    """(parts, keys of a part) of each request, as the kernels find them."""
    tile, splits, part, target = plan[:4]
    step = 256
    total = np.float32(0)
    for t, k in zip(tiles, keys):
        total = np.float32(total + np.float32(t) * np.float32(k))
    share = min(float(np.float32(total / np.float32(target))), 2.0 ** 30)
    most = max((int(share) + step) // step * step, part)
    parts = [min(max(-(-k // most), 1), splits) for k in keys]
    return [(p, -(-(-(-k // p)) // step) * step) for k, p in zip(keys, parts)]


def test_every_key_of_every_tile_is_dealt_out(plans):
    r = random.Random(3)
    cases = []
    for _ in range(1500):
        batch = r.choice((1, 1, 2, 3, 8, 30, 64))
        longest = int(2 ** r.uniform(0, 17))
        new = [r.choice((0, 1, 1, 5, r.randint(1, 900))) for _ in range(batch)]
        held = [r.randint(0, longest) for _ in range(batch)]
        tail = r.choice((0, 0, 3, 200))
        heads, group = r.choice(((1, 1), (1, 16), (2, 8), (8, 4), (12, 1), (3, 5)))
        cases.append((new, held, tail, heads, group, r.choice((64, 128))))
    asked = [(sum(n) + tail, g, h, len(n), max(m), d) for n, m, tail, h, g, d in cases]
    for (new, held, tail, heads, group, dim), ask, plan in zip(cases, asked, plans(asked)):
        tile, splits, part, target, bound, _ = plan
        assert target >= 1 and 1 <= splits <= 256 and part % 256 == 0
        tiles = [-(-n * group // tile) for n in new]
        keys = [m if n else 0 for n, m in zip(new, held)]
        count = -(-tail * group // tile)
        for t, k, (p, length) in zip(tiles, keys, parts_of(keys, tiles, plan)):
            assert p <= splits and p * length >= k, (ask, plan, k, p, length)
            count += t * p
        assert count <= bound, (ask, plan, count)


def test_more_requests_go_by_the_host(plans):
    for plan in plans([(65, 4, 8, 65, 8000, 128), (4000, 4, 8, 65, 8000, 128)]):
        assert plan[3] == 0 and plan[4] == 0


def test_workloads(plans):
    """Single tokens of 64 requests, of one; drafts; four long texts; chunks beside single tokens; a
    whole prompt, whose tiles fill the card."""
    got = plans([(64, 4, 8, 64, 8000, 128), (1, 4, 8, 1, 700, 128), (80, 4, 4, 16, 6000, 64),
                 (4, 8, 2, 4, 120000, 128), (1616, 4, 8, 6, 16000, 128),
                 (4096, 4, 8, 1, 4096, 128)])
    assert [p[:4] for p in got] == [(16, 15, 512, 96), (16, 1, 512, 62), (32, 11, 512, 192),
                                    (16, 234, 512, 249), (128, 16, 512, 64), (128, 1, 512, 64)]


def test_the_workspace_of_many_rows_is_bounded(plans):
    r = random.Random(5)
    cases = [(r.randint(500, 60000), 4, r.choice((1, 8)), r.randint(1, 10), r.randint(1, 200000), 128)
             for _ in range(300)]
    for (tokens, group, heads, *_), plan in zip(cases, plans(cases)):
        tile, splits, other = plan[0], plan[1], plan[5]
        assert tile == 128
        assert splits <= max(other, 1) or \
            (splits <= 16 and splits * tokens * group * heads * 128 * 4 <= 512 << 20)
