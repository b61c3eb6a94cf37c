"""What the sequence calls may touch, for every type and width: wrong offsets and lengths leave the
memory around each output and workspace as it was, and what lies in neighbours, behind the last
sequence and in unused rows of pages reaches nothing."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged import Case as Paged
from tests.test_gpu_seq import Case

import paper_2607_22696_amd as dsa

pytestmark = pytest.mark.gpu

KINDS = (("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128))
MARGIN = 1 << 16  # bytes before and behind


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dsa.load()
    yield


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Guards:
    """Tensors between margins of one value."""

    def __init__(self):
        self.held = []

    def __call__(self, shape, dtype, value=None):
        size = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        room = torch.full((size + 2 * MARGIN,), 0xA5, dtype=torch.uint8, device="cuda")
        t = room[MARGIN:MARGIN + size].view(dtype).view(shape)
        if value is not None:
            t.copy_(value)
        self.held.append(room)
        return t

    def check(self):
        torch.cuda.synchronize()
        for room in self.held:
            assert (room[:MARGIN] == 0xA5).all() and (room[-MARGIN:] == 0xA5).all()


def wrong_offsets(count, rows):
    """Offsets of `count` sequences: past the rows, negative, falling, none."""
    r = np.random.default_rng(count)
    far = r.integers(-2 ** 31, 2 ** 31 - 1, (3, count + 1))
    near = r.integers(-5, rows + 40, (3, count + 1))
    back = np.linspace(rows, 0, count + 1)[None].astype(np.int64)
    return np.concatenate([far, near, back, np.full((1, count + 1), rows), far * 0])


@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("count", (3, 70))
@pytest.mark.parametrize("causal", (False, True))
def test_wrong_offsets(dtype, D, count, causal):
    c = Case(240, [50, 260, 40] + [3] * (count - 3), H=4, KH=2, D=D, dtype=dtype, causal=causal,
             bias=(8, 20, True))
    rows, t = c.q.shape[0], c.q.dtype
    for cu in wrong_offsets(count, rows):
        guard = Guards()
        out, lse = guard(c.q.shape, t), guard(c.q.shape[:2], torch.float32)
        res = guard(c.q.shape, t) if dtype == "bf16" else None
        c.cu_q = ints(cu)
        print(f"  {cu[:4]}", flush=True)
        c.forward(out=out, lse=lse, out_res=res, need_residual=True)
        desc = dsa.make_seq_desc(count, rows, rows, 4, 2, D, causal, dtype, 0.0, c.rel_min,
                                 len(c.bucket), 8)
        grads = [guard(x.shape, x.dtype) for x in (c.q, c.k, c.v, c.how["rel_table"])]
        c.backward(out, res, lse, grads=grads, workspace=guard(
            (dsa.dsa3d_seq_backward_workspace_size(desc),), torch.uint8))
        guard.check()


@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("new", ([3, 4] + [1] * 70, [70, 4, 100]))
def test_wrong_lengths_offsets_and_pages(dtype, D, new):
    """Pages that the table does not name stay as they are."""
    count = len(new)
    c = Paged(250, new, [n + 60 for n in new], D=D, dtype=dtype, tail=3, spare=5,
              bias=(8, 20, False))
    rows, t = c.q.shape[0], c.q.dtype
    r = np.random.default_rng(3)
    k, v = c.q[:, :2].contiguous(), c.q[:, 2:4].contiguous()
    for i, cu in enumerate(wrong_offsets(count, rows)):
        held = r.integers(-2 ** 31, 2 ** 31 - 1, count) if i % 2 else np.asarray(c.held)
        pages = c.pages.copy()
        if i % 3 == 0:
            pages[:, 1] = r.integers(-2 ** 31, 2 ** 31 - 1, count)
        print(f"  {cu[:4]} {held[:4]}", flush=True)
        guard = Guards()
        out, lse = guard(c.q.shape, t), guard(c.q.shape[:2], torch.float32)
        desc = dsa.make_paged_desc(count, rows, 8, 2, D, c.kp.shape[0], 16, pages.shape[1],
                                   dtype=dtype, rel_min=c.rel_min, rel_span=len(c.bucket),
                                   rel_buckets=8)
        need = dsa.dsa3d_paged_forward_workspace_size(desc)
        dsa.paged_forward(c.q, c.kp, c.vp, ints(pages), ints(held), ints(cu), need_lse=True,
                          out=out, lse=lse, workspace=guard((need,), torch.uint8), **c.how)
        kp, vp = guard(c.kp.shape, t, c.kp), guard(c.vp.shape, t, c.vp)
        dsa.paged_append(k, v, kp, vp, ints(pages), ints(held), ints(cu))
        guard.check()
        free = torch.tensor(np.setdiff1d(np.arange(c.kp.shape[0]), pages)).cuda()
        assert len(free) >= 5
        assert torch.equal(kp[free], c.kp[free]) and torch.equal(vp[free], c.vp[free])


@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("empty", (0, 64))
def test_rows_of_others(dtype, D, causal, empty):
    """NaN and infinities in a neighbour and behind the last sequence leave the others' bits."""
    c = Case(260, [40, 200, 30] + [0] * empty, tail=70, H=4, KH=2, D=D, dtype=dtype, causal=causal,
             bias=(32, 128, True))
    first = c.forward(need_residual=True)
    grads = c.backward(first[0], first[2], first[1])
    for x in (c.q, c.k, c.v, c.g):
        x[270:] = float("nan")
        x[40:240, :, ::3] = float("inf")
        x[41:240:7] = float("nan")
    second = c.forward(need_residual=True)
    again = c.backward(second[0], second[2], second[1])
    for a, b in zip([*first, *grads[:3]], [*second, *again[:3]]):
        if a is not None:
            assert torch.equal(a[:40], b[:40]) and torch.equal(a[240:270], b[240:270])
    assert (second[0][270:] == 0).all() and torch.isneginf(second[1][270:]).all()
    assert all((x[270:] == 0).all() for x in again[:3])


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("new", ([1, 1, 1], [60, 1, 70]))
def test_unused_rows_of_pages(dtype, new):
    """As the test of 64 channels: NaN and infinities behind a request's last token, in spare pages
    and behind bad page numbers, at 128 channels."""
    c = Paged(270, new, [400, 170, 90], dtype=dtype, D=128, H=4, KH=2)
    c.pages[0, 3], c.pages[1, 0], c.pages[2, 1] = -1, c.kp.shape[0], -2 ** 31
    used = np.zeros(c.k64.shape[:2], bool)
    for b, m in enumerate(c.held):
        for j in range(m):
            if 0 <= c.pages[b, j // 16] < len(used):
                used[c.pages[b, j // 16], j % 16] = True
    free = torch.tensor(~used).cuda()
    c.kp[free] = float("nan")
    c.vp[free] = float("inf")
    c.check()
