"""Attention over a paged cache and the write into it on the GPU, against the float64 formulas
(oracle/sequence.py) within bounds derived in seq_util.py; and a prompt read and written on
through all the sequence calls together."""
import numpy as np
import pytest
import torch

from oracle import sequence as ref
from tests.seq_util import Bounds, near, rounded

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


class Case:
    def __init__(self, seed, new, held, H=8, KH=2, D=64, page=16, dtype="bf16", bias=None, tail=0,
                 spare=3, columns=0, causal=True, max_kv=0, fused=False):
        r = np.random.default_rng(seed)
        self.new, self.held, self.causal, self.max_kv = new, held, causal, max_kv
        counts = [-(-m // page) for m in held]
        num = sum(counts) + spare
        order = r.permutation(num)
        self.pages = np.full((len(held), max(counts + [1]) + columns), -1)
        at = 0
        for b, c in enumerate(counts):
            self.pages[b, :c] = order[at:at + c]
            at += c
        self.q, self.q64 = rounded(r, (sum(new) + tail, H, D), dtype, 1.5)
        kp, self.k64 = rounded(r, (num, page, KH, D), dtype)
        vp, self.v64 = rounded(r, (num, page, KH, D), dtype)
        self.q, self.kp, self.vp = self.q.cuda(), kp.cuda(), vp.cuda()
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
        return dsa.paged_forward(self.q, self.kp, self.vp, ints(self.pages), ints(self.held),
                                 ints(ref.starts(self.new)), self.causal, max_kv=self.max_kv,
                                 need_lse=True, **self.how, **kw)

    def check(self):
        out, lse = self.run()
        torch.cuda.synchronize()
        o, l, mag = ref.paged(self.q64, self.k64, self.v64, self.pages, self.held, self.new,
                              self.causal, None, self.table, self.bucket, self.rel_min)
        size, KH = self.k64.shape[1], self.k64.shape[2]
        k = np.concatenate([ref.gather(self.k64, self.v64, self.pages[b], m)[0]
                            for b, m in enumerate(self.held)] + [np.zeros((0, *self.k64.shape[2:]))])
        bd = Bounds(self.dtype, False, self.q64, k, self.new, self.held, 0.0, self.table)
        near("out", out, o, bd.out(o, mag))
        near("lse", lse, l, bd.lse(l))
        return out, lse


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
    "long_parts": dict(new=[1, 1, 2], held=[2600, 5, 1400], H=4, KH=2),
    "chunks": dict(new=[130, 1, 64, 300], held=[700, 650, 64, 301], H=4, KH=2),
    "chunks_128": dict(new=[150, 33], held=[1500, 33], H=8, KH=4, D=128),
    "chunk_of_odd_group": dict(new=[77, 50], held=[177, 60], H=6, KH=2, page=48),
    "whole_group": dict(new=[40, 1], held=[90, 900], H=16, KH=1),
    "rows_behind": dict(new=[3, 50], held=[60, 80], tail=140),
    "columns_behind": dict(new=[1, 1], held=[60, 80], columns=300),
    "not_causal": dict(new=[5, 60], held=[70, 80], causal=False),
    "strided": dict(new=[1, 40], held=[70, 80], fused=True),
}


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("name", CASES)
def test_paged_attention(name, dtype):
    Case(20 + len(name), dtype=dtype, **CASES[name]).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new,bias", [([1, 1, 2], (32, 128, False)), ([150, 3, 60], (32, 128, True)),
                                      ([1, 4, 1], (6, 5, True))])
def test_paged_bias(new, bias, dtype):
    Case(50 + len(new), new, [900, 40, 200], bias=bias, dtype=dtype, D=128).check()


def test_the_largest_bias():
    Case(54, [1, 30], [300, 200], H=16, KH=1, bias=(32, 128, True)).check()


@pytest.mark.parametrize("new", ([1, 1], [100, 1]))
def test_max_kv(new):
    """A bound that fits changes the parts, not the meaning; tokens behind a smaller one are not
    attended to."""
    a = Case(55, new, [3000, 1100], max_kv=3000, columns=4000)
    a.check()
    b = Case(56, new, [500, 90], max_kv=128)
    out, lse = b.run()
    torch.cuda.synchronize()
    b.pages[0, 128 // 16:] = -1  # what the bound hides, as pages without tokens
    o, l, mag = ref.paged(b.q64, b.k64, b.v64, b.pages, b.held, b.new, True)
    bd = Bounds("bf16", False, b.q64, b.k64.reshape(-1, *b.k64.shape[2:]), b.new, [128, 90], 0.0)
    bd.dt *= 4  # the bound above looked at other pairs than these
    near("out", out, o, bd.out(o, mag) * 2)
    near("lse", lse, l, bd.lse(l) * 2)


@pytest.mark.parametrize("new", ([1, 1, 1], [60, 1, 70]))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_bad_page_numbers_and_uninitialised_rows(new, dtype):
    """Page numbers outside the tensors hide their tokens; NaN in rows behind a request's last
    token, in spare pages and in page 0 behind them reach nothing."""
    c = Case(57, new, [400, 170, 90], dtype=dtype, page=16)
    c.pages[0, 3], c.pages[0, 11], c.pages[1, 0] = -1, 10 ** 6, c.kp.shape[0]
    c.pages[2, 1] = -2 ** 31
    used = np.zeros(c.k64.shape[:2], bool)
    for b, m in enumerate(c.held):
        for j in range(m):
            if 0 <= c.pages[b, j // 16] < len(used):
                used[c.pages[b, j // 16], j % 16] = True
    free = torch.tensor(~used).cuda()
    c.kp[free] = float("nan")
    c.vp[free] = float("inf")
    c.check()


def test_every_page_bad():
    c = Case(58, [1, 40], [50, 60])
    c.pages[:] = -1
    out, lse = c.run()
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_wrong_lengths_and_offsets_stay_inside():
    c = Case(59, [3, 4], [60, 70], tail=3)
    for held, cu in (([10 ** 9, -7], [0, 3, 7]), ([2 ** 31 - 1, 2 ** 31 - 1], [0, 3, 7]),
                     ([60, 70], [0, 900, -4])):
        out, lse = dsa.paged_forward(c.q, c.kp, c.vp, ints(c.pages), ints(held), ints(cu),
                                     need_lse=True)
        before = c.kp.clone()
        dsa.paged_append(c.q[:, :2].contiguous(), c.q[:, 2:4].contiguous(), before, before.clone(),
                         ints(c.pages), ints(held), ints(cu))
        torch.cuda.synchronize()


APPEND = {
    "single_tokens": dict(new=[1] * 5, held=[1, 16, 17, 40, 100]),
    "chunks": dict(new=[70, 0, 33, 1], held=[90, 12, 33, 300]),
    "odd_pages": dict(new=[20, 9], held=[50, 31], page=7),
    "rows_behind": dict(new=[5, 2], held=[30, 8], tail=9),
    "more_new_than_held": dict(new=[6, 2], held=[4, 0]),
}


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("strided", (False, True))
@pytest.mark.parametrize("name", APPEND)
def test_append(name, strided, dtype):
    c = Case(70 + len(name), dtype=dtype, H=2, KH=2, **APPEND[name])
    if name == "chunks":
        c.pages[0, 4], c.pages[3, 18] = -1, 10 ** 6
    r = np.random.default_rng(3)
    n = c.q.shape[0]
    (k, k64), (v, v64) = (rounded(r, (n, 2, 64), dtype) for _ in range(2))
    k, v = k.cuda(), v.cuda()
    if strided:
        both = torch.cat([k.flatten(1), v.flatten(1)], 1)
        k, v = both[:, :128].unflatten(1, (2, 64)), both[:, 128:].unflatten(1, (2, 64))
    want = ref.append(k64, v64, c.k64, c.v64, c.pages, c.held, c.new)
    dsa.paged_append(k, v, c.kp, c.vp, ints(c.pages), ints(c.held), ints(ref.starts(c.new)))
    torch.cuda.synchronize()
    assert np.array_equal(c.kp.double().cpu().numpy(), want[0])
    assert np.array_equal(c.vp.double().cpu().numpy(), want[1])


@pytest.mark.parametrize("new", ([1, 1, 1, 1], [90, 1, 300, 2]))
def test_same_bits_on_another_stream_and_replayed(new):
    c = Case(80, new, [3100, 700, 900, 64], H=8, KH=2, D=128)
    pages, held, cu = ints(c.pages), ints(c.held), ints(ref.starts(new))
    call = lambda **kw: dsa.paged_forward(c.q, c.kp, c.vp, pages, held, cu, need_lse=True, **kw)  # noqa: E731
    first = call()
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
    for most in (c.held, [2000, 650, 800, 60], c.held):
        held.copy_(ints(most))
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, third))


def test_a_prompt_read_in_chunks_and_written_on():
    """A biased causal sequence read whole by seq_forward equals the same tokens appended and
    attended to chunk by chunk and then token by token, within two calls' bounds."""
    r = np.random.default_rng(81)
    lengths, H, KH, D, page = [150, 40], 8, 2, 64, 16
    total = sum(lengths)
    (q, q64), (k, k64), (v, v64) = (rounded(r, (total, n, D), "bf16") for n in (H, KH, KH))
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    rel_buckets, rel_min = dsa.relative_buckets(32, 128, both=False)
    how = dict(rel_table=torch.tensor(r.standard_normal((32, H)), dtype=torch.float32).cuda(),
               rel_buckets=rel_buckets, rel_min=rel_min)
    whole, lse, _ = dsa.seq_forward(q, k, v, ints(ref.starts(lengths)), causal=True, **how)
    pages = r.permutation(20)[:14].reshape(2, 7)
    pages = np.concatenate([pages, np.full((2, 4), -1)], 1)
    pages[0, 7:10] = [x for x in range(20) if x not in pages][:3]
    kp = torch.full((20, page, KH, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    vp = kp.clone()
    got, got_l = torch.zeros_like(whole), torch.zeros_like(lse)
    done = [0, 0]
    for step in ([100, 38], [0, 1], [47, 0], [1, 1], [1, 0], [1, 0]):
        at = [ref.starts(lengths)[b] + done[b] for b in (0, 1)]
        rows = np.concatenate([np.arange(a, a + n) for a, n in zip(at, step)])
        done = [a + n for a, n in zip(done, step)]
        args = (ints(pages), ints(done), ints(ref.starts(step)))
        pick = torch.tensor(rows).cuda()
        dsa.paged_append(k[pick], v[pick], kp, vp, *args)
        got[pick], got_l[pick] = dsa.paged_forward(q[pick], kp, vp, *args, need_lse=True, **how)
    assert done == lengths
    table = how["rel_table"].double().cpu().numpy()
    o, l, mag = ref.forward(q64, k64, v64, lengths, lengths, True, None, table,
                            rel_buckets.tolist(), rel_min)
    bd = Bounds("bf16", False, q64, k64, lengths, lengths, 0.0, table)
    for a, b in ((whole, lse), (got, got_l)):
        near("out", a, o, bd.out(o, mag))
        near("lse", b, l, bd.lse(l))


@pytest.mark.parametrize("new", ([1, 2], [100, 1]))
def test_pages_past_32_bits(new):
    """Pages that lie 5 GB and more into their tensors: the write finds them, and attention gives
    the bits that it gives for the same pages in small tensors."""
    H, KH, D, page, far = 4, 2, 128, 16, 660_000
    c = Case(140, new, [700, 90], H=H, KH=KH, D=D, page=page)
    want = c.run()
    kp, vp = (torch.empty(far + c.kp.shape[0], page, KH, D, dtype=torch.bfloat16, device="cuda")
              for _ in range(2))
    assert kp.numel() > 2 ** 31 and kp[:far].numel() * 2 > 5 << 30
    kp[far:], vp[far:] = c.kp, c.vp
    small, c.kp, c.vp = (c.kp, c.vp), kp, vp
    near_pages = c.pages
    c.pages = np.where(near_pages >= 0, near_pages + far, -1)
    got = c.run()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    k, v = (torch.randn(sum(new), KH, D, device="cuda").bfloat16() for _ in range(2))
    rest = (ints(c.held), ints(ref.starts(new)))
    dsa.paged_append(k, v, *small, ints(near_pages), *rest)
    dsa.paged_append(k, v, kp, vp, ints(c.pages), *rest)
    assert torch.equal(kp[far:], small[0]) and torch.equal(vp[far:], small[1])


def test_two_graphs_with_one_workspace():
    cases = [Case(150 + i, new, held, H=8, KH=2, D=128)
             for i, (new, held) in enumerate((([1, 1, 1], [3000, 40, 900]),
                                              ([60, 1], [2100, 4000])))]
    room = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    graphs = []
    for c in cases:
        args = (c.q, c.kp, c.vp, ints(c.pages), ints(c.held), ints(ref.starts(c.new)))
        want = dsa.paged_forward(*args, need_lse=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = dsa.paged_forward(*args, need_lse=True, workspace=room)
        graphs.append((graph, held, want, args))
    for i in (0, 1, 1, 0, 0, 1):
        graph, held, want, _ = graphs[i]
        for x in held:
            x.fill_(float("nan"))
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_a_padded_batch():
    """Requests of no new tokens and rows behind the last request, as a batch of fixed size has
    them: the rows get 0 and -inf, the others what they get without the padding, and the write
    leaves the pages of requests without new tokens as they were."""
    c = Case(160, [1, 1, 0, 0], [200, 33, 50, 0], tail=2)
    out, lse = c.check()
    assert (out[2:] == 0).all() and torch.isneginf(lse[2:]).all()
    before = c.kp.clone()
    k = torch.randn(4, 2, 64, device="cuda").bfloat16()
    dsa.paged_append(k, k, c.kp, c.vp, ints(c.pages), ints(c.held), ints(ref.starts(c.new)))
    changed = (c.kp != before).flatten(2).any(-1).nonzero().tolist()
    assert sorted(changed) == sorted([[int(c.pages[0, 199 // 16]), 199 % 16],
                                      [int(c.pages[1, 32 // 16]), 32 % 16]])


@pytest.mark.parametrize("new", ([1, 2], [100, 1]))
def test_no_pages_and_no_columns(new):
    c = Case(180, new, [50, 60])
    args = (ints(c.held), ints(ref.starts(new)))
    k = c.q[:, :2].contiguous()
    for kp, vp, pages in ((c.kp[:0], c.vp[:0], ints(c.pages)),
                          (c.kp, c.vp, ints(np.zeros((2, 0))))):
        out, lse = dsa.paged_forward(c.q, kp, vp, pages, *args, need_lse=True)
        before = kp.clone()
        dsa.paged_append(k, k, kp, vp, pages, *args)
        assert (out == 0).all() and torch.isneginf(lse).all() and torch.equal(kp, before)
