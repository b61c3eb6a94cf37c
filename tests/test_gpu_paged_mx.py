"""The paged cache of 8 and 4 bits on the GPU: its write bit for bit and its reading exactly as
oracle/mx.py, attention over it against the float64 formulas (oracle/sequence.py) on the values that
the cache stands for, within the bounds of seq_util.py: the operands are exact, so that the kernels'
roundings are those of the attention over pages of the queries' type."""
import numpy as np
import pytest
import torch

from oracle import mx
from oracle import sequence as ref
from tests.seq_util import E32, TYPES, Bounds, near, rounded

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def table_of(r, held, page, num, columns=0):
    """Pages in no order, -1 behind a request's last."""
    counts = [-(-m // page) for m in held]
    order = r.permutation(num)
    pages = np.full((len(held), max(counts + [1]) + columns), -1)
    at = 0
    for b, c in enumerate(counts):
        pages[b, :c] = order[at:at + c]
        at += c
    return pages


def random_cache(r, num, page, KH, D, bits):
    """(tensors of a cache, values of its keys and of its values [num, page, KH, D])."""
    codes, scales, values = [], [], []
    for _ in range(2):
        x = r.standard_normal((num, KH, page, D)) * 2.0 ** r.integers(-2, 3, (num, KH, page, 1))
        c, s = mx.quantise(x, bits)
        codes.append(torch.tensor(mx.pack(c, bits)).cuda())
        scales.append(torch.tensor(s).cuda())
        values.append(mx.values(c, s, bits).transpose(0, 2, 1, 3))
    return (*codes, *scales), *values


class Case:
    def __init__(self, seed, new, held, H=8, KH=2, D=64, page=16, dtype="bf16", bits=8, bias=None,
                 tail=0, spare=3, columns=0, causal=True, max_kv=0, fused=False):
        r = np.random.default_rng(seed)
        self.new, self.held, self.causal, self.max_kv = new, held, causal, max_kv
        self.page, self.bits = page, bits
        num = sum(-(-m // page) for m in held) + spare
        self.pages = table_of(r, held, page, num, columns)
        self.q, self.q64 = rounded(r, (sum(new) + tail, H, D), dtype, 0.8)
        self.q = self.q.cuda()
        self.cache, self.k64, self.v64 = random_cache(r, num, page, KH, D, bits)
        if fused:
            wide = torch.zeros(self.q.shape[0], H * D + 64, dtype=self.q.dtype, device="cuda")
            wide[:, :H * D] = self.q.flatten(1)
            self.q = wide[:, :H * D].unflatten(1, (H, D))
        self.dtype, self.table, self.bucket, self.rel_min = dtype, None, None, 0
        self.how = {}
        if bias is not None:
            self.bucket, self.rel_min = dsa.dsa3d_relative_buckets(*bias)
            t = r.standard_normal((bias[0], H)).astype(np.float32)
            self.table = t.astype(np.float64)
            self.how = dict(rel_table=torch.tensor(t).cuda(), rel_buckets=ints(self.bucket),
                            rel_min=self.rel_min)

    def run(self, **kw):
        return dsa.paged_forward_mx(self.q, self.cache, ints(self.pages), ints(self.held),
                                    ints(ref.starts(self.new)), self.causal, max_kv=self.max_kv,
                                    need_lse=True, **self.how, **kw)

    def want(self):
        o, l, mag = ref.paged(self.q64, self.k64, self.v64, self.pages, self.held, self.new,
                              self.causal, None, self.table, self.bucket, self.rel_min)
        k = np.concatenate([ref.gather(self.k64, self.v64, self.pages[b], m)[0]
                            for b, m in enumerate(self.held)] + [np.zeros((0, *self.k64.shape[2:]))])
        bd = Bounds(self.dtype, False, self.q64, k, self.new, self.held, 0.0, self.table)
        return o, l, bd.out(o, mag), bd.lse(l)

    def check(self):
        out, lse = self.run()
        torch.cuda.synchronize()
        o, l, out_bound, lse_bound = self.want()
        near("out", out, o, out_bound)
        near("lse", lse, l, lse_bound)
        return out, lse


# ----------------------------------------------------------------------------- write and read

def wide_numbers(r, shape, dtype):
    """Blocks of every size: normal numbers times powers of two over the type's whole range, zeros,
    numbers half way between elements, and some blocks that are not finite or nearly too large."""
    x = r.standard_normal(shape)
    flat = x.reshape(-1, 32)
    flat *= 2.0 ** r.integers(-135, 125, (len(flat), 1))
    some = r.permutation(len(flat))
    few = max(1, len(flat) // 12)
    flat[some[:few]] = 0.0
    flat[some[few:2 * few], ::3] *= -0.0
    flat[some[2 * few:4 * few]] = r.integers(-56, 57, (2 * few, 32)) * 2.0 ** r.integers(-60, 60)
    flat[some[4 * few:5 * few], 7] = np.inf
    flat[some[5 * few:6 * few], 31] = np.nan
    flat[some[6 * few:7 * few]] = r.uniform(2.8e38, 3.389e38, (few, 32))
    flat[some[7 * few:8 * few]] *= 2.0 ** r.integers(-12, 1, (few, 32))
    t = torch.tensor(np.clip(x, -3.389e38, 3.389e38) if not np.isinf(x).any() else
                     np.where(np.isinf(x), x, np.clip(x, -3.389e38, 3.389e38))).to(TYPES[dtype])
    return t, t.double().numpy()


APPEND = {
    "single_tokens": dict(new=[1] * 5, held=[1, 16, 17, 40, 100]),
    "chunks": dict(new=[70, 0, 33, 1], held=[90, 12, 33, 300]),
    "odd_pages": dict(new=[20, 9], held=[50, 31], page=7),
    "rows_behind": dict(new=[5, 2], held=[30, 8], tail=9),
    "more_new_than_held": dict(new=[6, 2], held=[4, 0]),
    "one_narrow_head": dict(new=[3, 1, 0, 6], held=[5, 1, 9, 60], KH=1),
    "three_heads": dict(new=[2, 9], held=[30, 9], KH=3),
    "eight_wide_heads": dict(new=[1, 4], held=[33, 4], KH=8, D=128),
    "one_wide_head": dict(new=[1, 4, 1], held=[33, 4, 1], KH=1, D=128, page=1),
    "70_requests": dict(new=[1, 0] * 35, held=[1 + 13 * b % 90 for b in range(70)]),
    "many_steps": dict(new=[1900, 1, 1400], held=[1900, 7, 1450], KH=3, D=128, page=24),
}


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("name", APPEND)
def test_write_and_read(name, dtype, bits):
    how = dict(KH=2, D=64, page=16, tail=0)
    how.update(APPEND[name])
    new, held, KH, D, page = (how[n] for n in ("new", "held", "KH", "D", "page"))
    r = np.random.default_rng(70 + len(name))
    num = sum(-(-m // page) for m in held) + 3
    pages = table_of(r, held, page, num)
    if name == "chunks":
        pages[0, 4], pages[3, 18] = -1, 10 ** 6
    rows = sum(new) + how["tail"]
    (k, k64), (v, v64) = (wide_numbers(r, (rows, KH, D), dtype) for _ in range(2))
    k, v = k.cuda(), v.cuda()
    if name in ("chunks", "three_heads"):  # slices of a fused projection
        both = torch.cat([k.flatten(1), v.flatten(1)], 1)
        k, v = both[:, :KH * D].unflatten(1, (KH, D)), both[:, KH * D:].unflatten(1, (KH, D))
    cache = tuple(torch.randint(0, 256, t.shape, dtype=torch.uint8).cuda()
                  for t in dsa.paged_cache_mx(num, page, KH, D, bits, device="cpu"))
    want = [t.cpu().numpy().copy() for t in cache]
    back = np.zeros((2, rows, KH, D))
    for i, x in enumerate((k64, v64)):
        code, scale = mx.quantise(x, bits)
        value, code = mx.values(code, scale, bits), mx.pack(code, bits)
        for row, p, at in mx.places(pages, held, new, page, num):
            want[i][p, :, at], want[2 + i][p, :, at] = code[row], scale[row]
            back[i, row] = value[row]
    rest = (ints(pages), ints(held), ints(ref.starts(new)))
    dsa.paged_append_mx(k, v, cache, *rest)
    torch.cuda.synchronize()
    for got, w, what in zip(cache, want, ("k", "v", "k_scales", "v_scales")):
        got = got.cpu().numpy()
        bad = np.argwhere(got != w)
        assert not len(bad), (what, len(bad), bad[0], got[tuple(bad[0])], w[tuple(bad[0])])
    for other in ("bf16", "f32"):
        got = dsa.paged_read_mx(cache, *rest, rows, TYPES[other])
        for g, w in zip(got, back):
            assert g.dtype == TYPES[other]
            assert np.array_equal(g.double().cpu().numpy(), w, equal_nan=True)


@pytest.mark.parametrize("bits", (8, 4))
def test_every_element_and_power(bits):
    """All codes with all scale bytes that stand for values of normal bf16 numbers, and 255."""
    codes = np.arange(256, dtype=np.uint8).reshape(4, 64) if bits == 8 else \
        np.tile(np.arange(256, dtype=np.uint8), 2).reshape(16, 32)[:8]
    tokens = [(row, s) for s in [*range(10, 246), 255] for row in codes]
    n = len(tokens)
    held = np.stack([t[0] for t in tokens])
    scale = np.repeat(np.array([[t[1]] for t in tokens], np.uint8), 2, 1)
    cache = dsa.paged_cache_mx(1, n, 1, 64, bits)
    for i, x in enumerate((held, held, scale, scale)):
        cache[i].copy_(torch.tensor(x).view(1, 1, n, -1))
    want = mx.values(mx.unpack(held, bits), scale, bits)
    for dtype in TYPES.values():
        got = dsa.paged_read_mx(cache, ints([[0]]), ints([n]), ints([0, n]), n, dtype)
        for g in got:
            assert np.array_equal(g[:, 0].double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("bits", (8, 4))
def test_reading_earlier_tokens_into_given_rows(bits):
    """Tokens 20 .. 59 of 90 by a smaller length, into rows of wider tensors; rows behind the last
    request are cleared, what lies between rows is left."""
    r = np.random.default_rng(5)
    cache, k64, v64 = random_cache(r, 9, 16, 2, 64, bits)
    pages = r.permutation(9)[:6][None]
    k, v = (torch.full((43, 160), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = [x[:, :128].unflatten(1, (2, 64)) for x in (k, v)]
    got = dsa.paged_read_mx(cache, ints(pages), ints([60]), ints([0, 40]), 43, k=rows[0], v=rows[1])
    assert got[0].data_ptr() == k.data_ptr()
    for g, x, wide in zip(got, (k64, v64), (k, v)):
        want = np.zeros((43, 2, 64))
        want[:40] = [x[pages[0, j // 16], j % 16] for j in range(20, 60)]
        assert np.array_equal(g.double().cpu().numpy(), want)
        assert (wide[:, 128:] == 7.0).all()


def test_no_rows_no_pages_no_columns():
    cache, _, _ = random_cache(np.random.default_rng(6), 4, 16, 2, 64, 8)
    none = tuple(t[:0] for t in cache)
    x = torch.ones(3, 2, 64, device="cuda")
    q = torch.ones(3, 4, 64, device="cuda")
    for c, pages in ((none, ints([[0, 1], [2, 3]])), (cache, ints(np.zeros((2, 0))))):
        args = (pages, ints([20, 9]), ints([0, 1, 3]))
        before = [t.clone() for t in c]
        dsa.paged_append_mx(x, x, c, *args)
        assert all(torch.equal(a, b) for a, b in zip(c, before))
        assert all((t == 0).all() for t in dsa.paged_read_mx(c, *args, 3, torch.float32))
        out, lse = dsa.paged_forward_mx(q, c, *args, need_lse=True)
        assert (out == 0).all() and torch.isneginf(lse).all()
    args = (ints([[0, 1], [2, 3]]), ints([20, 9]), ints([0, 0, 0]))
    dsa.paged_append_mx(x[:0], x[:0], cache, *args)
    assert dsa.paged_read_mx(cache, *args, 0)[0].shape == (0, 2, 64)
    assert dsa.paged_forward_mx(q[:0], cache, *args)[0].shape == (0, 4, 64)


# ----------------------------------------------------------------------------- attention

CASES = {
    "one_token": dict(new=[1], held=[1]),
    "one_request": dict(new=[1], held=[700], H=4, KH=1, D=128),
    "single_tokens": dict(new=[1] * 9, held=[1, 2, 15, 16, 17, 127, 128, 129, 500]),
    "pages_end_inside_tiles": dict(new=[1, 1, 3], held=[100, 33, 50], page=7),
    "one_row_pages": dict(new=[2, 1], held=[40, 150], page=1),
    "large_pages": dict(new=[1, 5], held=[300, 77], page=256, H=2, KH=2),
    "few_rows_over_a_tile": dict(new=[9, 1, 5], held=[200, 3, 5], H=12, KH=3),
    "no_new_tokens": dict(new=[0, 2, 0], held=[30, 40, 0]),
    "more_new_than_held": dict(new=[4, 3], held=[2, 0]),
    "long_parts": dict(new=[1, 1, 2], held=[2600, 5, 1400], H=4, KH=2, D=128),
    "chunks": dict(new=[130, 1, 64, 300], held=[700, 650, 64, 301], H=4, KH=2),
    "chunks_128": dict(new=[150, 33], held=[1500, 33], H=8, KH=4, D=128),
    "chunk_of_odd_group": dict(new=[77, 50], held=[177, 60], H=6, KH=2, page=48),
    "whole_group": dict(new=[40, 1], held=[90, 900], H=16, KH=1),
    "rows_behind": dict(new=[3, 50], held=[60, 80], tail=140),
    "columns_behind": dict(new=[1, 1], held=[60, 80], columns=300),
    "not_causal": dict(new=[5, 60], held=[70, 80], causal=False),
    "strided": dict(new=[1, 40], held=[70, 80], fused=True),
}


LONGER = {
    # requests that a wave holds a lane each, with lengths of every class, and one more than that
    "64_requests": dict(new=[1] * 64, held=[1 + 37 * b % 1900 for b in range(64)]),
    "65_requests": dict(new=[1] * 65, held=[1 + 37 * b % 1900 for b in range(65)]),
    "none_of_64": dict(new=[0, 1] * 32, held=[(53 * b) % 700 for b in range(64)], tail=5),
    "many_parts": dict(new=[1, 1], held=[70000, 2001], H=2, KH=1, D=128, page=100),
    "drafts_128": dict(new=[6, 5, 0, 7, 6, 3], held=[3000, 700, 50, 65, 2100, 33], D=128),
    "drafts_64": dict(new=[6, 5, 0, 7, 6, 3], held=[3000, 700, 50, 65, 2100, 33], page=24),
    "66_chunks": dict(new=[30] * 66, held=[30 + 31 * b for b in range(66)], KH=1, H=4),
    "chunks_in_parts": dict(new=[100, 3, 1, 40], held=[9000, 700, 2600, 41], KH=1, H=4, D=128),
    "tiles_and_parts": dict(new=[9, 1, 40] + [1] * 13, held=[3000, 5000, 1200] + [20] * 13, KH=1),
}


@pytest.mark.parametrize("bits,dtype", ((8, "bf16"), (4, "bf16"), (4, "f32")))
@pytest.mark.parametrize("name", LONGER)
def test_dealt_out(name, bits, dtype):
    Case(20 + len(name), dtype=dtype, bits=bits, **LONGER[name]).check()


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("name", CASES)
def test_attention(name, dtype, bits):
    Case(20 + len(name), dtype=dtype, bits=bits, **CASES[name]).check()


@pytest.mark.parametrize("bits,D", ((8, 128), (4, 64)))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new,bias", [([1, 1, 2], (32, 128, False)), ([150, 3, 60], (32, 128, True)),
                                      ([1, 4, 1], (6, 5, True)), ([6, 5, 7], (32, 128, False))])
def test_bias(new, bias, dtype, bits, D):
    Case(50 + len(new), new, [900, 40, 200], bias=bias, dtype=dtype, D=D, bits=bits).check()


def test_the_largest_bias():
    Case(54, [1, 30], [300, 200], H=16, KH=1, bias=(32, 128, True)).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new", ([1, 1], [60, 3]))
def test_a_bias_that_hides(new, dtype):
    """-inf and the lowest float in the table hide their distances; a row may see nothing."""
    c = Case(53, new, [60, 30], bias=(8, 16, False), dtype=dtype)
    t = c.how["rel_table"]
    t[0] = -torch.inf          # a query's own key
    t[3, 1:3] = torch.finfo(torch.float32).min
    t[:, 4] = -torch.inf       # all of a head's
    c.table = t.double().cpu().numpy()
    out, lse = c.check()
    assert (out[:, 4] == 0).all() and torch.isneginf(lse[:, 4]).all()


@pytest.mark.parametrize("new", ([1, 1], [100, 1]))
def test_max_kv(new):
    """A bound that fits changes the parts, not the meaning; tokens behind a smaller one are not
    attended to."""
    Case(55, new, [3000, 1100], max_kv=3000, columns=4000).check()
    b = Case(56, new, [500, 90], max_kv=128)
    out, lse = b.run()
    b.pages[0, 128 // 16:] = -1  # what the bound hides, as pages without tokens
    o, l, out_bound, lse_bound = b.want()
    near("out", out, o, out_bound)
    near("lse", lse, l, lse_bound)


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("new", ([1, 1, 1], [60, 1, 70]))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_bad_page_numbers_and_uninitialised_rows(new, dtype, bits):
    """Page numbers outside the tensors hide their tokens; NaN in rows behind a request's last
    token, in spare pages and in page 0 behind them reach nothing."""
    c = Case(57, new, [400, 170, 90], dtype=dtype, bits=bits)
    num = c.k64.shape[0]
    c.pages[0, 3], c.pages[0, 11], c.pages[1, 0] = -1, 10 ** 6, num
    c.pages[2, 1] = -2 ** 31
    used = np.zeros((num, 16), bool)
    for b, m in enumerate(c.held):
        for j in range(m):
            if 0 <= c.pages[b, j // 16] < num:
                used[c.pages[b, j // 16], j % 16] = True
    free = torch.tensor(~used).cuda()[:, None, :, None]
    for t in c.cache:
        t.masked_fill_(free, 255)
    c.check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new", ([1, 1], [70, 1]))
def test_a_block_that_is_not_finite(new, dtype):
    """A NaN block among a request's keys or values makes NaN of the rows that see it (a value's in
    its channels), and nothing of another request's."""
    for which in (0, 1):
        c = Case(63, new, [150, 90], dtype=dtype, H=4, KH=2)
        want = c.run()[0]
        c.cache[2 + which][c.pages[0, 2], 1, 5, 1] = 255  # token 37 of request 0, head 1
        out, lse = c.run()
        n = new[0]
        assert torch.equal(out[n:], want[n:]) and torch.equal(out[:n, :2], want[:n, :2])
        hit = out[:n, 2:] if which == 0 else out[:n, 2:, 32:]
        assert torch.isnan(hit).all()
        if which == 0:
            assert torch.isnan(lse[:n, 2:]).all()


@pytest.mark.parametrize("new", ([1, 1, 2], [70, 1, 20]))
def test_requests_that_share_pages(new):
    """A common beginning is held once; a page may stand twice in a table."""
    c = Case(64, new, [300, 200, 180], H=8, KH=2, D=128, bits=4)
    c.pages[1, :6] = c.pages[0, :6]
    c.pages[2, :6] = c.pages[0, :6]
    c.pages[2, 7] = c.pages[2, 6]
    c.check()


@pytest.mark.parametrize("new,H,KH", (([1] * 64, 288, 9), ([1, 1], 2, 1), ([40], 4, 1)))
def test_a_long_text_of_repeated_pages(new, H, KH):
    """204,800 tokens that stand in 16 pages, 800 times each: attention is that over 256 tokens, lse
    larger by log 800.  More parts than a wave has lanes, also where there are many rows to join."""
    held = [256] + [5] * (len(new) - 1)
    c = Case(65, new, held, H=H, KH=KH, bits=4, causal=False)
    o, l, out_bound, lse_bound = c.want()
    more = 800 * 256 * E32  # the terms of the sums
    one = c.pages[0, :16]
    c.pages = np.concatenate([c.pages, np.full((len(new), 800 * 16 - c.pages.shape[1]), -1)], 1)
    c.pages[0], c.held = np.tile(one, 800), [800 * 256] + held[1:]
    out, lse = c.run()
    l[:new[0]] += np.log(800)
    mag = np.abs(c.v64[c.pages[0, :16]]).max()
    near("out", out, o, out_bound + 2 * more * mag)
    near("lse", lse, l, lse_bound + 2 * more + np.abs(l) * 4 * E32)


def test_every_page_bad():
    for new in ([1, 1], [1, 40]):
        c = Case(58, new, [50, 60])
        c.pages[:] = -1
        out, lse = c.run()
        assert (out == 0).all() and torch.isneginf(lse).all()


def test_wrong_lengths_and_offsets_stay_inside():
    c = Case(59, [3, 4], [60, 70], tail=3)
    x = c.q[:, :2].contiguous()
    for held, cu in (([10 ** 9, -7], [0, 3, 7]), ([2 ** 31 - 1, 2 ** 31 - 1], [0, 3, 7]),
                     ([60, 70], [0, 900, -4])):
        args = (ints(c.pages), ints(held), ints(cu))
        dsa.paged_forward_mx(c.q, c.cache, *args, need_lse=True)
        dsa.paged_read_mx(c.cache, *args, 10)
        dsa.paged_append_mx(x, x, tuple(t.clone() for t in c.cache), *args)
        torch.cuda.synchronize()


@pytest.mark.parametrize("new", ([1, 1, 1, 1], [90, 1, 300, 2]))
def test_same_bits_on_another_stream_and_replayed(new):
    c = Case(80, new, [3100, 700, 900, 64], H=8, KH=2, D=128, bits=4)
    pages, held, cu = ints(c.pages), ints(c.held), ints(ref.starts(new))
    x = torch.randn(sum(new), 2, 128, device="cuda").bfloat16()

    def call(cache=c.cache, **kw):
        dsa.paged_append_mx(x, x, cache, pages, held, cu)
        k, v = dsa.paged_read_mx(cache, pages, held, cu, sum(new))
        out = dsa.paged_forward_mx(c.q, cache, pages, held, cu, need_lse=True, **kw)
        return (*out, k, v, *cache)

    first = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(out=torch.full_like(first[0], float("nan")),
                      workspace=torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda"))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = call()
    start = [t.clone() for t in c.cache]
    for most in (c.held, [2000, 650, 800, 60], c.held):
        held.copy_(ints(most))
        for t, s in zip(c.cache, start):
            t.copy_(s)
        want = [t.clone() for t in call()]
        for t, s in zip(c.cache, start):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, third))


def test_two_graphs_with_one_workspace():
    cases = [Case(150 + i, new, held, H=8, KH=2, D=128)
             for i, (new, held) in enumerate((([1, 1, 1], [3000, 40, 900]),
                                              ([60, 1], [2100, 4000])))]
    room = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    graphs = []
    for c in cases:
        args = (c.q, c.cache, ints(c.pages), ints(c.held), ints(ref.starts(c.new)))
        want = dsa.paged_forward_mx(*args, need_lse=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = dsa.paged_forward_mx(*args, need_lse=True, workspace=room)
        graphs.append((graph, held, want, args))
    for i in (0, 1, 1, 0, 0, 1):
        graph, held, want, _ = graphs[i]
        for x in held:
            x.fill_(float("nan"))
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.parametrize("bits", (8, 4))
@pytest.mark.parametrize("new", ([1, 2], [100, 1]))
def test_pages_past_32_bits(new, bits):
    """Pages that lie 5 GB and more into their tensors: write and read find them, and attention
    gives the bits that it gives for the same pages in small tensors."""
    H, KH, D, page = 4, 2, 128, 16
    far = (5 << 30) // (KH * page * D * bits // 8) + 1
    c = Case(140, new, [700, 90], H=H, KH=KH, D=D, page=page, bits=bits)
    want = c.run()
    small, far_pages = c.cache, np.where(c.pages >= 0, c.pages + far, -1)
    large = tuple(torch.empty(far + t.shape[0], *t.shape[1:], dtype=torch.uint8, device="cuda")
                  for t in small)
    assert large[0][:far].numel() > 5 << 30
    for a, b in zip(large, small):
        a[far:] = b
    near_pages, c.cache, c.pages = c.pages, large, far_pages
    assert all(torch.equal(a, b) for a, b in zip(want, c.run()))
    k, v = (torch.randn(sum(new), KH, D, device="cuda") for _ in range(2))
    rest = (ints(c.held), ints(ref.starts(new)))
    dsa.paged_append_mx(k, v, small, ints(near_pages), *rest)
    dsa.paged_append_mx(k, v, large, ints(far_pages), *rest)
    assert all(torch.equal(a[far:], b) for a, b in zip(large, small))
    for a, b in zip(dsa.paged_read_mx(small, ints(near_pages), *rest, sum(new)),
                    dsa.paged_read_mx(large, ints(far_pages), *rest, sum(new))):
        assert torch.equal(a, b)


def test_a_padded_batch():
    """Requests of no new tokens and rows behind the last request, as a batch of fixed size has
    them: the rows get 0 and -inf, the others what they get without the padding, and the write
    leaves the pages of requests without new tokens as they were."""
    c = Case(160, [1, 1, 0, 0], [200, 33, 50, 0], tail=2)
    out, lse = c.check()
    assert (out[2:] == 0).all() and torch.isneginf(lse[2:]).all()
    before = [t.clone() for t in c.cache]
    k = torch.randn(4, 2, 64, device="cuda").bfloat16()
    dsa.paged_append_mx(k, k, c.cache, ints(c.pages), ints(c.held), ints(ref.starts(c.new)))
    changed = (c.cache[0] != before[0]).any(-1).any(1).nonzero().tolist()
    assert sorted(changed) == sorted([[int(c.pages[0, 199 // 16]), 199 % 16],
                                      [int(c.pages[1, 32 // 16]), 32 % 16]])


@pytest.mark.parametrize("bits", (8, 4))
def test_a_prompt_read_in_chunks_and_written_on(bits):
    """A biased causal sequence: seq_forward over the keys and values as the cache holds them
    (written, then read back) equals attention over the cache, chunk by chunk and then token by
    token, each within its bounds of the same formulas."""
    r = np.random.default_rng(81)
    lengths, H, KH, D, page = [150, 40], 8, 2, 64, 16
    total = sum(lengths)
    q, q64 = rounded(r, (total, H, D), "bf16")
    (k, k64), (v, v64) = (rounded(r, (total, KH, D), "bf16") for _ in range(2))
    q, k, v, starts = q.cuda(), k.cuda(), v.cuda(), ints(ref.starts(lengths))
    rel_buckets, rel_min = dsa.relative_buckets(32, 128, both=False)
    how = dict(rel_table=torch.tensor(r.standard_normal((32, H)), dtype=torch.float32).cuda(),
               rel_buckets=rel_buckets, rel_min=rel_min)
    pages = table_of(r, lengths, page, 20, 2)
    cache = dsa.paged_cache_mx(20, page, KH, D, bits)
    for t in cache:
        t.fill_(255)
    got, got_l = torch.zeros_like(q), torch.zeros(total, H, device="cuda")
    done = [0, 0]
    for step in ([100, 38], [0, 1], [47, 0], [1, 1], [1, 0], [1, 0]):
        at = [ref.starts(lengths)[b] + done[b] for b in (0, 1)]
        pick = torch.tensor(np.concatenate([np.arange(a, a + n) for a, n in zip(at, step)])).cuda()
        done = [a + n for a, n in zip(done, step)]
        args = (ints(pages), ints(done), ints(ref.starts(step)))
        dsa.paged_append_mx(k[pick], v[pick], cache, *args)
        got[pick], got_l[pick] = dsa.paged_forward_mx(q[pick], cache, *args, need_lse=True, **how)
    assert done == lengths
    kb, vb = dsa.paged_read_mx(cache, ints(pages), ints(lengths), starts, total)
    whole, lse, _ = dsa.seq_forward(q, kb, vb, starts, causal=True, **how)
    k64, v64 = (mx.values(*mx.quantise(x, bits), bits) for x in (k64, v64))
    assert np.array_equal(kb.double().cpu().numpy(), k64)
    assert np.array_equal(vb.double().cpu().numpy(), v64)
    table = how["rel_table"].double().cpu().numpy()
    o, l, mag = ref.forward(q64, k64, v64, lengths, lengths, True, None, table,
                            rel_buckets.tolist(), rel_min)
    bd = Bounds("bf16", False, q64, k64, lengths, lengths, 0.0, table)
    for a, b in ((whole, lse), (got, got_l)):
        near("out", a, o, bd.out(o, mag))
        near("lse", b, l, bd.lse(l))
