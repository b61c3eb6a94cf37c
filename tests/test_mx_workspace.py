"""The room that paged_forward_mx asks for its partial results: no more than the parts that are dealt
out can fill, however long a cache the call allows, and enough for all of them."""
import random
import subprocess

import pytest

import paper_2607_22696_amd as dsa
from tests.test_paged_mx_rules import HDR, parts_of

PROGRAM = r"""
#include <cstdio>
#include "paged_rules.h"
int main() {
  long tokens;
  int group, heads, batch, most, dim;
  while (scanf("%ld %d %d %d %d %d", &tokens, &group, &heads, &batch, &most, &dim) == 6) {
    const dsa3d::MxPlan p = dsa3d::paged_mx_plan(tokens, group, heads, batch, most, dim);
    printf("%d %d %d %d %ld %ld\n", p.tile, p.splits, p.part, p.target, (long)p.bound,
           (long)p.room);
  }
}
"""


@pytest.fixture(scope="module")
def rooms(tmp_path_factory):
    d = tmp_path_factory.mktemp("mx_workspace")
    src, exe = d / "r.cpp", d / "r"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", HDR, str(src), "-o", str(exe)])

    def ask(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.check_output([str(exe)], input=text, text=True)
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def need(tokens, heads, kv_heads, batch, most, head_dim=128, bits=8):
    page = 64
    d = dsa.make_paged_desc(batch, tokens, heads, kv_heads, head_dim, 4, page, -(-most // page), most)
    return dsa.dsa3d_paged_forward_mx_workspace_size(d, bits)


MIB = 1 << 20


@pytest.mark.parametrize("tokens,heads,kv_heads,batch,most,limit", (
    (64 * 5, 32, 8, 64, 131072, 30), (64 * 8, 32, 8, 64, 131072, 30),
    (64 * 32, 32, 32, 64, 131072, 60), (64, 32, 8, 64, 131072, 15),
    (1616, 32, 8, 6, 16000, 80), (1616, 32, 8, 6, 131072, 80), (64 * 32, 128, 128, 64, 131072, 120)))
def test_calls_with_long_page_tables(tokens, heads, kv_heads, batch, most, limit):
    assert 0 < need(tokens, heads, kv_heads, batch, most) <= limit * MIB


def test_it_does_not_grow_with_the_longest_cache():
    """From where every part has its least length on, at any rows per workgroup."""
    r = random.Random(11)
    for _ in range(300):
        batch = r.choice((1, 2, 7, 30, 64))
        heads, kv_heads = r.choice(((1, 1), (16, 1), (16, 16), (32, 8), (128, 8), (64, 64)))
        tokens = batch * r.choice((1, 1, 2, 5, 8, 30, 200))
        # 768 workgroups with parts at a time; 8 parts per key head beside twice as many; 128 rows of
        # 129 numbers
        tile = 128 if tokens * (heads // kv_heads) > 32 * batch else 32
        parts = (2 * max(512 if tile == 128 else 768, kv_heads) + 8 * kv_heads) * tile
        for most in (3000, 40000, 1 << 20, 1 << 30):
            got = need(tokens, heads, kv_heads, batch, most)
            assert got <= tokens * heads * 16 + parts * 129 * 4 + 1024, \
                (tokens, heads, kv_heads, batch, most, got)


def test_every_part_has_room(rooms):
    r = random.Random(4)
    cases = []
    for _ in range(1500):
        batch = r.choice((1, 1, 2, 3, 8, 30, 64))
        longest = int(2 ** r.uniform(0, 18))
        new = [r.choice((0, 1, 1, 5, r.randint(1, 900))) for _ in range(batch)]
        held = [r.choice((r.randint(0, longest), longest)) for _ in range(batch)]
        heads, group = r.choice(((1, 1), (1, 16), (2, 8), (8, 4), (12, 1), (3, 5)))
        wide = r.choice((1, 1, 3, 50))  # the page table may allow more than is held
        cases.append((new, held, (sum(new), group, heads, batch, max(held) * wide, 128)))
    some = 0
    for (new, held, ask), plan in zip(cases, rooms([c[2] for c in cases])):
        tiles = [-(-n * ask[1] // plan[0]) for n in new]
        keys = [m if n else 0 for n, m in zip(new, held)]
        dealt = [t * p for t, (p, _) in zip(tiles, parts_of(keys, tiles, plan)) if p > 1]
        assert sum(dealt) <= plan[5] <= plan[4], (ask, plan, sum(dealt))
        some += bool(dealt)
    assert some > 300


def test_more_requests_have_the_room_of_the_bf16_cache(rooms):
    """Beyond 64 requests parts are not dealt out, and go by rows as there."""
    assert rooms([(70, 4, 8, 70, 8000, 128)])[0][3:] == (0, 0, 0)
    d = dsa.make_paged_desc(70, 70, 32, 8, 128, 4, 64, 125, 8000)
    other = dsa.dsa3d_paged_forward_workspace_size(d)
    assert other > 0
    assert need(70, 32, 8, 70, 8000) <= other + 70 * 32 * 16 + 1024
