"""Attention of packed sequences and its relative position bias on the GPU, forward and backward,
against the float64 formulas (oracle/sequence.py) within bounds derived in seq_util.py."""
import numpy as np
import pytest
import torch

from oracle import sequence as ref
from tests.seq_util import TYPES, Bounds, near, rounded

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


class Case:
    """Tensors of one case on the GPU and in float64, and the calls on them."""

    def __init__(self, seed, lengths, keys=None, H=2, KH=2, D=64, dtype="bf16", causal=False,
                 scale=0.0, bias=None, tail=0, table_edit=None, fused=False):
        r = np.random.default_rng(seed)
        self.lengths, self.own = lengths, keys is None
        self.keys = lengths if keys is None else keys
        self.dtype, self.causal, self.scale = dtype, causal, scale
        nq, nk = sum(lengths) + tail, sum(self.keys) + tail
        self.q, self.q64 = rounded(r, (nq, H, D), dtype, 1.5)
        self.k, self.k64 = rounded(r, (nk, KH, D), dtype)
        self.v, self.v64 = rounded(r, (nk, KH, D), dtype)
        self.g, self.g64 = rounded(r, (nq, H, D), dtype)
        self.q, self.k, self.v, self.g = (x.cuda() for x in (self.q, self.k, self.v, self.g))
        if fused:  # slices of one projection's rows
            both = torch.cat([x.flatten(1) for x in (self.q, self.k, self.v)], 1)
            parts = both.split([H * D, KH * D, KH * D], 1)
            self.q, self.k, self.v = (p.unflatten(1, (n, D))
                                      for p, n in zip(parts, (H, KH, KH)))
        cu = lambda x: torch.tensor(ref.starts(x), dtype=torch.int32).cuda()  # noqa: E731
        self.cu_q, self.cu_k = cu(lengths), None if self.own else cu(self.keys)
        self.table = self.bucket = None
        self.rel_min = 0
        self.how = {}
        if bias is not None:
            self.bucket, self.rel_min = dsa.dsa3d_relative_buckets(*bias)
            self.table = r.standard_normal((bias[0], H)).astype(np.float32)
            if table_edit is not None:
                table_edit(self.table, self.bucket)
            self.how = dict(rel_table=torch.tensor(self.table).cuda(), rel_min=self.rel_min,
                            rel_buckets=torch.tensor(self.bucket, dtype=torch.int32).cuda())
            self.table = self.table.astype(np.float64)
        self.ref = dict(causal=causal, scale=scale or None, table=self.table, bucket=self.bucket,
                        rel_min=self.rel_min)

    def forward(self, **kw):
        return dsa.seq_forward(self.q, self.k, self.v, self.cu_q, self.cu_k, self.causal,
                               self.scale, **self.how, **kw)

    def backward(self, out, res, lse, **kw):
        return dsa.seq_backward(self.q, self.k, self.v, out, res, lse, self.g, self.cu_q,
                                self.cu_k, self.causal, self.scale, **self.how, **kw)

    def check(self, residual=False, backward=True):
        out, lse, res = self.forward(need_residual=residual)
        torch.cuda.synchronize()
        residual = residual and self.dtype == "bf16"
        bd = Bounds(self.dtype, residual, self.q64, self.k64, self.lengths, self.keys, self.scale,
                    self.table)
        o, l, mag = ref.forward(self.q64, self.k64, self.v64, self.lengths, self.keys, **self.ref)
        near("out", out, o, bd.out(o, mag))
        near("lse", lse, l, bd.lse(l))
        if residual:
            near("out + out_res", out.double() + res.double(), o, bd.read_out(o, mag))
        else:
            assert res is None
        if not backward:
            return
        got = self.backward(out, res, lse)
        torch.cuda.synchronize()
        want, mags, extra = ref.backward(self.q64, self.k64, self.v64, self.g64, self.lengths,
                                         self.keys, out_error=bd.read_out(o, mag), **self.ref)
        for name, a, b, limit in zip(("dq", "dk", "dv", "d_rel_table"), got, want,
                                     bd.grads(want, mags, extra)):
            near(name, a, b, limit)
        assert len(got) == (3 if self.table is None else 4)


PLAIN = {
    "one_token": dict(lengths=[1]),
    "short_prompts": dict(lengths=[1, 37, 5, 64, 20], H=3, KH=3),
    "empty_sequences": dict(lengths=[0, 5, 0, 0, 130, 1, 0]),
    "tile_edges": dict(lengths=[31, 32, 33, 63, 64, 65, 127, 128, 129, 257]),
    "groups_128": dict(lengths=[70, 200, 3], H=8, KH=2, D=128),
    "one_key_head": dict(lengths=[140, 9], H=5, KH=1),
    "longer_keys": dict(lengths=[40, 1, 130], keys=[300, 129, 131], H=4, KH=2),
    "fewer_keys": dict(lengths=[130, 40, 7], keys=[3, 0, 70], H=2, KH=1),
    "no_keys_at_all": dict(lengths=[3, 40], keys=[0, 0]),
    "no_queries": dict(lengths=[0, 0], keys=[3, 140]),
    "many_sequences": dict(lengths=[(7 * i) % 5 for i in range(150)], H=2, KH=1),
    "rows_behind": dict(lengths=[33, 100], tail=75, H=2, KH=2),
    "fused_projection": dict(lengths=[100, 61], H=4, KH=2, fused=True),
    "scale": dict(lengths=[90, 5], scale=0.31),
}


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("name", PLAIN)
def test_packed_sequences(name, causal, dtype):
    Case(10 + len(name), causal=causal, dtype=dtype, **PLAIN[name]).check()


@pytest.mark.parametrize("causal", (False, True))
def test_float32_of_128_channels(causal):
    Case(40, [65, 160, 1], H=4, KH=2, D=128, dtype="f32", causal=causal).check()


def test_residual_without_a_bias():
    Case(41, [65, 160, 1], H=2, KH=1, D=128, causal=True).check(residual=True)


def hide_own(table, bucket):
    table[0] = -np.inf  # distance 0


def hide_all(table, bucket):
    table[:, 0] = np.finfo(np.float32).min
    table[:, 1:] = -np.inf


def some_without(table, bucket):
    bucket[3], bucket[5] = -1, len(table)


BIAS = {
    "both_ways": dict(lengths=[200, 1, 77, 300], bias=(32, 128, True)),
    "behind_only": dict(lengths=[200, 1, 77, 300], bias=(32, 128, False), causal=True),
    "ahead_shares_a_bucket": dict(lengths=[150, 40], bias=(8, 20, False)),
    "near_span": dict(lengths=[257, 64], bias=(6, 5, True), H=4, KH=2, D=128),
    "wide_span": dict(lengths=[300, 20], bias=(64, 1000, True)),
    "groups": dict(lengths=[150, 131], bias=(16, 64, True), H=8, KH=2, causal=True),
    "other_keys": dict(lengths=[70, 20], keys=[160, 150], bias=(32, 128, True), causal=True),
    "own_place_hidden": dict(lengths=[5, 140], bias=(8, 20, True), table_edit=hide_own),
    "own_place_hidden_causal": dict(lengths=[5, 140], bias=(8, 20, False), causal=True,
                                    table_edit=hide_own),
    "everything_hidden": dict(lengths=[5, 70], bias=(8, 20, True), table_edit=hide_all),
    "distances_without_a_bucket": dict(lengths=[50, 70], bias=(8, 20, True),
                                       table_edit=some_without),
    "most_buckets": dict(lengths=[180], bias=(256, 900, True), H=1, KH=1),
}


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("name", BIAS)
def test_relative_bias(name, dtype):
    Case(60 + len(name), dtype=dtype, **BIAS[name]).check(residual=True)


def test_bias_gradient_without_residual_and_left_out():
    c = Case(90, [200, 33], bias=(32, 128, True))
    c.check(residual=False)
    out, lse, res = c.forward(need_residual=True)
    a, b = c.backward(out, res, lse), c.backward(out, res, lse, need_table=False)
    assert b[3] is None and all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


@pytest.mark.parametrize("causal", (False, True))
def test_rows_of_others_reach_nothing(causal):
    """NaN and infinities behind the last sequence and in a neighbour leave a sequence's results
    as they are, bit for bit, and rows behind the last sequence get 0 and -inf."""
    c = Case(91, [40, 100, 30], tail=70, H=4, KH=2, causal=causal, bias=(32, 128, True))
    first = c.forward(need_residual=True)
    grads = c.backward(first[0], first[2], first[1])
    for x in (c.q, c.k, c.v, c.g):
        x[170:] = float("nan")
        x[40:140, :, ::3] = float("inf")
    second = c.forward(need_residual=True)
    again = c.backward(second[0], second[2], second[1])
    for a, b in zip(list(first) + list(grads[:3]), list(second) + list(again[:3])):
        assert torch.equal(a[:40], b[:40]) and torch.equal(a[140:170], b[140:170])
    assert (second[0][170:] == 0).all() and torch.isneginf(second[1][170:]).all()
    assert all((x[170:] == 0).all() for x in again[:3])


def test_same_bits_again_on_another_stream_and_into_given_tensors():
    c = Case(92, [300, 129, 64], H=4, KH=2, D=128, causal=True, bias=(32, 128, False))
    out, lse, res = c.forward(need_residual=True)
    grads = c.backward(out, res, lse)
    torch.cuda.synchronize()
    fill = lambda x: torch.full_like(x, float("nan"))  # noqa: E731
    into = [fill(x) for x in (out, lse, res)]
    given = [fill(x) for x in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.forward(need_residual=True, out=into[0], lse=into[1], out_res=into[2])
        c.backward(into[0], into[2], into[1], grads=given,
                   workspace=torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda"))
    side.synchronize()
    for a, b in zip([out, lse, res, *grads], into + given):
        assert torch.equal(a, b)


def test_a_captured_step_replays():
    c = Case(93, [150, 70], H=2, KH=1, causal=True, bias=(32, 128, False))
    eager = c.forward(need_residual=True)
    grads = c.backward(eager[0], eager[2], eager[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = c.forward(need_residual=True)
        hgrads = c.backward(held[0], held[2], held[1])
    for scale in (1.0, 0.5, 1.0):
        c.q.copy_(torch.from_numpy(c.q64 * scale).to(TYPES["bf16"]))
        want = c.forward(need_residual=True)
        want_g = c.backward(want[0], want[2], want[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([*want, *want_g], [*held, *hgrads]):
            assert torch.equal(a, b)
    for a, b in zip([*eager, *grads], [*held, *hgrads]):
        assert torch.equal(a, b)


def test_wrong_offsets_stay_inside_the_tensors():
    """Offsets past the rows, negative or falling: results are undefined, other memory is not
    touched."""
    c = Case(94, [50, 60, 40], H=2, KH=1)
    guard = torch.full((150 + 64, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for cu in ([0, 90, 30, 1000], [0, -5, 2_000_000_000, 10], [0, 0, 0, 0], [77, 80, 90, 150]):
        c.cu_q = torch.tensor(cu, dtype=torch.int32).cuda()
        out, lse, _ = c.forward(out=guard[32:182])
        c.backward(out, None, lse)
        torch.cuda.synchronize()
        assert (guard[:32] == 7).all() and (guard[182:] == 7).all()


LONG = {
    "long_128": dict(lengths=[700, 270], H=4, KH=2, D=128),
    "long_64": dict(lengths=[700, 270], H=3, KH=1),
    "long_biased": dict(lengths=[700, 270], H=4, KH=2, D=128, bias=(32, 128, True)),
    "long_other_keys": dict(lengths=[300, 520], keys=[650, 400], H=2, KH=2, D=128),
}


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("name", LONG)
def test_runs_of_whole_tiles(name, causal, dtype):
    """Sequences of many tiles, most of them seen whole."""
    Case(100 + len(name), causal=causal, dtype=dtype, **LONG[name]).check(residual=True)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_the_widest_bias(dtype, D):
    """The most distances a bias can tell apart, forward and backward."""
    c = Case(110, [150, 40], H=2, KH=1, D=D, dtype=dtype, bias=(256, 1023, True))
    assert len(c.bucket) == dsa.DSA3D_SEQ_MAX_SPAN - 1
    c.check(residual=True)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("how", ("plain", "causal", "bias", "residual"))
def test_many_queries_of_long_sequences(how, D):
    """8,320 and 40 tokens of 16 heads, where the forward takes more queries at a time; some of
    the rows are compared."""
    lengths, H, KH = [8320, 40], 16, 4
    nq = sum(lengths)
    g = torch.Generator().manual_seed(D)
    q, k, v = (torch.randn(nq, n, D, generator=g).bfloat16().cuda() for n in (H, KH, KH))
    cu = torch.tensor(ref.starts(lengths), dtype=torch.int32).cuda()
    causal, kw, table, bucket, rel_min = how != "plain", {}, None, None, 0
    if how == "bias":
        bucket, rel_min = dsa.dsa3d_relative_buckets(32, 128, False)
        table = torch.randn(32, H, generator=g)
        kw = dict(rel_table=table.cuda(), rel_min=rel_min,
                  rel_buckets=torch.tensor(bucket, dtype=torch.int32).cuda())
        table = table.double().numpy()
    out, lse, res = dsa.seq_forward(q, k, v, cu, causal=causal, need_residual=how == "residual",
                                    **kw)
    torch.cuda.synchronize()
    k64, v64 = (x.double().cpu().numpy() for x in (k, v))
    rows = [0, 1, 31, 32, 255, 256, 4000, 4127, 8191, 8192, 8300, 8319, 8320, 8359]
    q64 = q[rows].double().cpu().numpy()
    for i, row in enumerate(rows):  # a row alone, at the end of the keys that it sees
        first = 0 if row < 8320 else 8320
        last = row + 1 if causal else (8320 if row < 8320 else nq)
        args = ([1], [last - first])
        o, l, mag = ref.forward(q64[i:i + 1], k64[first:last], v64[first:last], *args, True
                                if how == "bias" else False, None, table, bucket, rel_min)
        bd = Bounds("bf16", how == "residual", q64[i:i + 1], k64[first:last], *args, 0.0, table)
        near("out", out[row:row + 1], o, bd.out(o, mag))
        near("lse", lse[row:row + 1], l, bd.lse(l))
        if res is not None:
            near("out + out_res", out[row:row + 1].double() + res[row:row + 1].double(), o,
                 bd.read_out(o, mag))


def test_rows_far_apart():
    """q, k and v as columns of one tensor whose rows lie 8 MB apart, 4.8 GB in all, give the bits
    of contiguous ones."""
    c = Case(120, [500, 100], H=2, KH=1, causal=True)
    wide = torch.empty(600, 1 << 22, dtype=torch.bfloat16, device="cuda")
    out, lse, _ = c.forward()
    grads = c.backward(out, None, lse)
    at = 0
    for name in ("q", "k", "v"):
        x = getattr(c, name)
        to = wide[:, at:at + x[0].numel()].unflatten(1, x.shape[1:])
        to.copy_(x)
        setattr(c, name, to)
        at += 1 << 20
    out2, lse2, _ = c.forward()
    for a, b in zip((out, lse, *grads), (out2, lse2, *c.backward(out2, None, lse2))):
        assert torch.equal(a, b)


def test_two_graphs_with_one_workspace():
    """Two captured backward passes that were given the same workspace, replayed in turn."""
    cases = [Case(130 + i, n, H=4, KH=2, D=128, causal=True, bias=(32, 128, False))
             for i, n in enumerate(([300, 64], [40, 290, 7]))]
    room = torch.empty(1 << 23, dtype=torch.uint8, device="cuda")
    held, want, graphs = [], [], []
    for c in cases:
        out, lse, res = c.forward(need_residual=True)
        want.append(c.backward(out, res, lse))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(c.backward(out, res, lse, workspace=room))
        graphs.append((graph, out, lse, res))
    for i in (0, 1, 1, 0, 0, 1):
        for x in held[i]:
            x.fill_(float("nan"))
        room.fill_(255)
        graphs[i][0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held[i], want[i]))


@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("count", (1, 2, 62, 63, 64, 65))
def test_numbers_of_sequences(count, causal):
    """Around the number of sequences that a wave holds, with lengths that rise, fall and repeat,
    empty ones among them, other keys than queries and rows behind the last sequence."""
    lengths = [(37 * i) % 301 if i % 5 else (0, 128, 300)[i // 5 % 3] for i in range(count)]
    keys = [(53 * i + 40) % 280 if i % 7 else 0 for i in range(count)]
    c = Case(170 + count, lengths, keys=keys, H=2, KH=1, causal=causal, tail=140,
             bias=(8, 20, True))
    c.check(residual=True)
