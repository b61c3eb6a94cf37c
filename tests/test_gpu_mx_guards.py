"""What the calls on an 8- or 4-bit cache may touch: margins around every output, the workspace of
exactly the size asked for and the cache stay as they were, at wrong offsets, lengths and page numbers
too; lengths beyond the page table and below 0 have their results."""
import numpy as np
import pytest
import torch

from oracle import sequence as ref
from tests.mx_forms import FORMS
from tests.seq_util import TYPES, near
from tests.test_gpu_paged_mx import Case, ints
from tests.test_gpu_seq_guards import KINDS, Guards, wrong_offsets

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


def need_of(c, pages):
    rows, H, D = c.q.shape
    num, KH = c.cache[0].shape[:2]
    how = {} if c.bucket is None else dict(rel_min=c.rel_min, rel_span=len(c.bucket),
                                           rel_buckets=len(c.table))
    d = dsa.make_paged_desc(len(c.new), rows, H, KH, D, num, c.page, pages.shape[1], c.max_kv,
                            c.causal, c.dtype, **how)
    return dsa.dsa3d_paged_forward_mx_workspace_size(d, c.bits)


def guarded(c, guard, pages, held, cu, fill=None):
    """paged_forward_mx into guarded tensors; the workspace starts as `fill` of its size."""
    out, lse = guard(c.q.shape, c.q.dtype), guard(c.q.shape[:2], torch.float32)
    need = need_of(c, pages)
    room = guard((need,), torch.uint8, None if fill is None else fill(need)) if need else None
    dsa.paged_forward_mx(c.q, c.cache, ints(pages), ints(held), ints(cu), c.causal,
                         max_kv=c.max_kv, need_lse=True, out=out, lse=lse, workspace=room, **c.how)
    return out, lse


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("name", ("few_rows_in_few_parts", "few_rows_in_many_parts", "drafts", "chunks",
                                  "66_drafts"))
def test_ordinary_calls(name, dtype, D, bits):
    c = Case(500 + len(name), D=D, bits=bits, dtype=dtype, **FORMS[name][0])
    guard = Guards()
    c.cache = tuple(guard(t.shape, torch.uint8, t) for t in c.cache)
    before = [t.clone() for t in c.cache]
    got = guarded(c, guard, c.pages, c.held, ref.starts(c.new))
    guard.check()
    for a, b in zip(got, c.run()):
        assert torch.equal(a, b)
    assert all(torch.equal(a, b) for a, b in zip(c.cache, before))


WRONG = {
    "single_tokens": dict(new=[1, 1, 2], held=[700, 300, 4], columns=70),
    "drafts": dict(new=[6, 5, 7], held=[700, 300, 4], columns=70),
    "chunks": dict(new=[70, 4, 100], held=[200, 60, 90], columns=70),
    "72_requests": dict(new=[3, 4] + [1] * 70, held=[1200, 60] + [20 + b for b in range(70)]),
}


@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("name", WRONG)
def test_wrong_lengths_offsets_and_pages(name, dtype, D):
    """Pages that the table does not name stay as they are.  The workspace starts as one value or
    as small numbers, which a row that is nobody's could take for where its parts are."""
    bits = 8 if D == 64 else 4
    c = Case(510 + len(name), D=D, dtype=dtype, bits=bits, tail=3, spare=5, bias=(8, 20, False),
             **WRONG[name])
    count, rows = len(c.new), c.q.shape[0]
    r = np.random.default_rng(3)
    k, v = c.q[:, :2].contiguous(), c.q[:, 2:4].contiguous()

    def small(size):
        x = torch.zeros((size + 3) // 4, dtype=torch.int32, device="cuda").random_(0, 40)
        return x.view(torch.uint8)[:size]

    for i, cu in enumerate(wrong_offsets(count, rows)):
        held = r.integers(-2 ** 31, 2 ** 31 - 1, count) if i % 2 else np.asarray(c.held)
        pages = c.pages.copy()
        if i % 3 == 0:
            pages[:, 1] = r.integers(-2 ** 31, 2 ** 31 - 1, count)
        print(f"  {cu[:4]} {held[:4]}", flush=True)
        guard = Guards()
        kept = c.cache
        c.cache = cache = tuple(guard(t.shape, torch.uint8, t) for t in kept)
        guarded(c, guard, pages, held, cu, small if i % 2 else None)
        guard.check()
        assert all(torch.equal(a, b) for a, b in zip(cache, kept))
        back = [guard((rows, 2, D), TYPES[dtype]) for _ in range(2)]
        dsa.paged_read_mx(cache, ints(pages), ints(held), ints(cu), rows, TYPES[dtype], *back)
        dsa.paged_append_mx(k, v, cache, ints(pages), ints(held), ints(cu))
        guard.check()
        free = torch.tensor(np.setdiff1d(np.arange(kept[0].shape[0]), pages)).cuda()
        assert len(free) >= 5
        assert all(torch.equal(a[free], b[free]) for a, b in zip(cache, kept))
        c.cache = kept


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new", ([1, 2], [6, 5], [70, 40], [1] * 70))
def test_lengths_beyond_the_page_table_and_below_zero(new, dtype, bits):
    """A request of more tokens than its table has columns for stands behind them all: its new
    tokens see every one that has a page.  One of a negative length holds none."""
    far, none = range(0, len(new), 2), range(1, len(new), 2)
    c = Case(520 + len(new), new, [800 if b < 2 else 40 for b in range(len(new))], dtype=dtype,
             bits=bits)
    most = c.pages.shape[1] * c.page
    held = np.zeros(len(new), np.int64)
    held[list(far)] = np.resize([2 ** 31 - 1, 10 ** 9, most + 1000], len(far))
    held[list(none)] = np.resize([-7, -2 ** 31], len(none))
    guard = Guards()
    out, lse = guarded(c, guard, c.pages, held, ref.starts(new))
    guard.check()
    c.held, c.causal = [most if b % 2 == 0 else 0 for b in range(len(new))], False
    o, l, out_bound, lse_bound = c.want()
    near("out", out, o, out_bound)
    near("lse", lse, l, lse_bound)


@pytest.mark.parametrize("name", ("single_tokens", "drafts", "chunks"))
@pytest.mark.parametrize("dtype,D", KINDS)
def test_lengths_that_change_after_the_capture(name, dtype, D):
    """The room is that of every length that the page table allows: a graph captured at short
    lengths and replayed at long ones stays within it and gives the eager call's bits."""
    new, most = {"single_tokens": ([1, 1, 1], [6000, 900, 2600]),
                 "drafts": ([6, 0, 7], [3000, 50, 2100]),
                 "chunks": ([100, 3, 40], [4000, 700, 2600])}[name]
    c = Case(530 + len(name), new, most, D=D, dtype=dtype, columns=300)
    pages, cu = ints(c.pages), ints(ref.starts(new))
    short = [n + 3 for n in new]
    held = ints(short)
    guard = Guards()
    out, lse = guard(c.q.shape, c.q.dtype), guard(c.q.shape[:2], torch.float32)
    room = guard((need_of(c, c.pages),), torch.uint8)

    def call(**kw):
        return dsa.paged_forward_mx(c.q, c.cache, pages, held, cu, need_lse=True, **kw)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, lse=lse, workspace=room)
    for lengths in (most, short, [m // 2 for m in most], most):
        held.copy_(ints(lengths))
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph.replay()
        guard.check()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("new,H", (([1] * 64, 2), ([9] * 64, 2), ([1] * 63 + [90], 4)))
@pytest.mark.parametrize("dtype,bits", (("bf16", 4), ("f32", 8)))
def test_64_requests_in_parts(new, H, dtype, bits):
    """As many parts as are dealt out: each request has 8,192 tokens that stand in the same 16 pages,
    32 times each, so that attention is that over 256 tokens and lse larger by log 32."""
    c = Case(540 + len(new), new, [256] + [1] * 63, H=H, KH=1, bits=bits, dtype=dtype, causal=False)
    c.pages = np.tile(c.pages[0, :16], (64, 1))
    c.held = [256] * 64
    o, l, out_bound, lse_bound = c.want()
    pages = np.tile(c.pages, (1, 32))
    guard = Guards()
    c.held, more = [8192] * 64, 8192 * 2.0 ** -23  # the terms of the sums
    out, lse = guarded(c, guard, pages, c.held, ref.starts(new))
    guard.check()
    l += np.log(32)
    near("out", out, o, out_bound + 2 * more * np.abs(c.v64[c.pages[0]]).max())
    near("lse", lse, l, lse_bound + 2 * more + np.abs(l) * 4 * 2.0 ** -23)
