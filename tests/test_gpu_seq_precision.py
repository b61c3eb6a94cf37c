"""What the bounds of tests/seq_util.py cannot see of the packed-sequence kernels: the table
gradient in float32 accuracy, from the call's own statistics and from those of more keys than the
call has; gradients of keys whose weights are small; float32 results and the parts of their
operands."""
import numpy as np
import pytest
import torch

from tests import seq_table
from tests.seq_util import TYPES, rounded
from tests.test_gpu_seq import Case

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


def of_the_bound(name, got, want, limit):
    worst = float((np.abs(got.double().cpu().numpy() - want) / limit).max())
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, (name, worst)


class Biased:
    """One sequence whose values share an offset, so that Delta and its rounding are large beside
    dS, and a bias of few distances, beyond which most pairs are."""

    def __init__(self, seed, n, dtype, D, causal, H=4, KH=2):
        r = np.random.default_rng(seed)
        self.dtype, self.causal, self.n = dtype, causal, n
        (self.q, self.q64), (self.k, self.k64), (self.g, self.g64) = (
            rounded(r, (n, heads, D), dtype, std) for heads, std in ((H, 1.5), (KH, 1.0), (H, 1.0)))
        v = r.standard_normal((n, KH, D)) + 6.0
        self.v = torch.tensor(v).to(TYPES[dtype])
        self.v64 = self.v.double().numpy()
        self.bucket, self.rel_min = dsa.dsa3d_relative_buckets(6, 5, not causal)
        self.table = r.standard_normal((6, H)).astype(np.float32)
        self.bias = dict(rel_table=torch.tensor(self.table).cuda(), rel_buckets=ints(self.bucket))
        self.table = self.table.astype(np.float64)
        self.place = (self.table, self.bucket, self.rel_min)
        self.q, self.k, self.v, self.g = (x.cuda() for x in (self.q, self.k, self.v, self.g))


@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("dtype,D", (("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)))
def test_the_table_gradient_in_float32_accuracy(dtype, D, causal):
    c = Biased(200 + D, 1100, dtype, D, causal)
    how = dict(causal=causal, rel_min=c.rel_min, **c.bias)
    out, lse, res = dsa.seq_forward(c.q, c.k, c.v, ints([0, c.n]), need_residual=True, **how)
    got = dsa.seq_backward(c.q, c.k, c.v, out, res, lse, c.g, ints([0, c.n]), **how)[3]
    o, l = seq_table.statistics(c.q64, c.k64, c.v64, *c.place, causal)
    of_the_bound("d_rel_table", got, *seq_table.table_gradient(
        c.q64, c.k64, c.v64, c.g64, o, l, *c.place, causal,
        carried=2.0 ** (-18 if dtype == "bf16" else -23)))


@pytest.mark.parametrize("residual", (True, False))
@pytest.mark.parametrize("dtype,D", (("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)))
def test_the_table_gradient_from_statistics_of_more_keys(dtype, D, residual):
    """Keys in two calls with the joined out and lse, as ranks that share a sequence's keys have
    them: dS = alpha (dP - Delta) of either call's keys, which do not add up to zero."""
    c = Biased(210 + D, 700, dtype, D, False)
    o, l = seq_table.statistics(c.q64, c.k64, c.v64, *c.place)
    out = torch.tensor(o).to(TYPES[dtype])
    res = (torch.tensor(o) - out.double()).bfloat16() if dtype == "bf16" and residual else None
    given = out.double().numpy() + (0.0 if res is None else res.double().numpy())
    lse = torch.tensor(l).float()
    half = c.n // 2
    for first, last in ((0, half), (half, c.n)):
        # key j of the call is key first + j of all, whose distance is less by what lies behind
        shift = last - c.n
        got = dsa.seq_backward(c.q, c.k[first:last], c.v[first:last], out.cuda(),
                               None if res is None else res.cuda(), lse.cuda(), c.g,
                               ints([0, c.n]), ints([0, last - first]), rel_min=c.rel_min - shift,
                               **c.bias)[3]
        of_the_bound("d_rel_table", got, *seq_table.table_gradient(
            c.q64, c.k64[first:last], c.v64[first:last], c.g64, given, lse.double().numpy(),
            *c.place, shift=shift))


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_keys_of_small_weights(dtype, D):
    """Weights down to e^-60 of a row's largest: dk and dv of their keys are as exact, relative
    to their own terms, as any."""
    c = Case(220, [200, 33], H=4, KH=2, D=D, dtype=dtype, scale=1.0)
    c.q[..., 0] = 1
    c.k[:] = 0
    c.k[..., 0] = -4.0 * (torch.arange(233) % 16)[:, None]
    c.q64, c.k64 = (x.double().cpu().numpy() for x in (c.q, c.k))
    c.check()


@pytest.mark.parametrize("D", (64, 128))
def test_the_parts_of_float32_operands(D):
    """x x - z, z being x x rounded: what a product loses stands alone.  Each operand is three
    bf16 parts to half a step, so that beside the products that are left out, at most 2^-24, the
    sum of two products and a third addend near 1 can lose 2^-24 for each; parts that are cut off
    would lose 2^-21 of these x."""
    x = 1 + 2.0 ** -7 - np.arange(1, 17) * 2.0 ** -23
    z = (x * x).astype(np.float32).astype(np.float64)
    q, k = torch.zeros(2, 16, 1, D, dtype=torch.float32)
    q[:, 0, 0], q[:, 0, 1] = torch.tensor(x), torch.tensor(-z)
    k[:, 0, 0], k[:, 0, 1] = torch.tensor(x), 1.0
    lse = dsa.seq_forward(q.cuda(), k.cuda(), k.cuda(), ints(range(17)), scale=1024.0)[1][:, 0]
    want = 1024 * (x * x - z)
    of_the_bound("lse", lse, want, 1024 * 4.25 * 2.0 ** -24 + np.abs(want) * 2.0 ** -21)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("causal", (False, True))
def test_float32_results(D, causal):
    """Root mean square errors against the spread that float32 roundings give (operands of two
    parts would be at 2.8 to 5.5 of it, see test_seq_table_bound.py); paged results too."""
    r = np.random.default_rng(230 + D)
    (q, q64), (k, k64), (v, v64), (g, g64) = (rounded(r, (300, 2, D), "f32", s)
                                              for s in (1.5, 1.0, 1.0, 1.0))
    q, k, v, g = (x.cuda() for x in (q, k, v, g))
    cu = ints([0, 300])
    out, lse, _ = dsa.seq_forward(q, k, v, cu, causal=causal)
    got = [out, *dsa.seq_backward(q, k, v, out, None, lse, g, cu, causal=causal)]
    want, spread = seq_table.spreads(q64, k64, v64, g64, causal)
    paged = [x.new_zeros(10, 32, 2, D) for x in (k, v)]
    table = ints(np.random.default_rng(1).permutation(10)[None])
    dsa.paged_append(k, v, *paged, table, ints([300]), cu)
    got.append(dsa.paged_forward(q, *paged, table, ints([300]), cu, causal=causal)[0])
    got.append(torch.cat([dsa.paged_forward(q[i:i + 1], *paged, table, ints([i + 1 if causal else
                          300]), ints([0, 1]), causal=causal)[0] for i in range(300)]))
    for name, a, i in zip(("out", "dq", "dk", "dv", "chunk", "tokens"), got, (0, 1, 2, 3, 0, 0)):
        ratio = seq_table.rms(a.double().cpu().numpy() - want[i]) / seq_table.rms(spread[i])
        print(f"  {name}: {ratio:.3f} of the spread", flush=True)
        assert ratio <= 2.0, (name, ratio)


@pytest.mark.parametrize("bits", (0x7fffffff, -1, 0x7f800001))
@pytest.mark.parametrize("D", (64, 128))
def test_a_nan_among_the_statistics_stays(D, bits):
    """lse of one query a NaN of any bits: its dq, and dk and dv of every key that it sees, are NaN
    in its head and its key head alone."""
    c = Case(280, [70], H=2, KH=2, D=D)
    out, lse, _ = c.forward()
    want = c.backward(out, None, lse)
    lse.view(torch.int32)[9, 1] = bits
    dq, dk, dv = c.backward(out, None, lse)
    assert dq[9, 1].isnan().all() and dk[:, 1].isnan().all() and dv[:, 1].isnan().all()
    dq[9, 1] = want[0][9, 1]
    for a, b in zip((dq, dk[:, :1], dv[:, :1]), (want[0], want[1][:, :1], want[2][:, :1])):
        assert torch.equal(a, b)
