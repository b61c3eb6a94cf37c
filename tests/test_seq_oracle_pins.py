"""Pins of the plain sequence attention (oracle/sequence.py) against torch: gradients by
differentiation in float64, the masks, empty rows, buckets by whole-number arithmetic."""
import numpy as np
import pytest
import torch

from oracle import sequence as ref

import paper_2607_22696_amd as dsa


def inputs(seed, lengths, keys, H, KH, D):
    r = np.random.default_rng(seed)
    return (r.standard_normal((sum(lengths), H, D)), r.standard_normal((sum(keys), KH, D)),
            r.standard_normal((sum(keys), KH, D)), r.standard_normal((sum(lengths), H, D)))


def torch_attention(q, k, v, table, lengths, keys, causal, bucket, rel_min):
    """One sequence at a time, heads together, -inf masks and torch's softmax."""
    outs, q0, k0 = [], 0, 0
    group = q.shape[1] // k.shape[1]
    for n, m in zip(lengths, keys):
        a = q[q0:q0 + n].transpose(0, 1)
        b, c = (x[k0:k0 + m].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
        t = a @ b.transpose(1, 2) / q.shape[2] ** 0.5
        d = torch.arange(m)[None] - (torch.arange(n)[:, None] + m - n)
        if table is not None:
            t = t + table[bucket[(d - rel_min).clamp(0, len(bucket) - 1)]].permute(2, 0, 1)
        if causal:
            t = t.masked_fill(d > 0, -torch.inf)
        outs.append((torch.softmax(t, -1) @ c).transpose(0, 1))
        q0, k0 = q0 + n, k0 + m
    return torch.cat(outs)


@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("biased", (False, True))
def test_forward_and_gradients_match_differentiation(causal, biased):
    lengths, keys = [5, 1, 9], [7, 4, 9]
    q, k, v, g = inputs(1, lengths, keys, 4, 2, 8)
    table = np.random.default_rng(2).standard_normal((6, 4)) if biased else None
    bucket, rel_min = dsa.dsa3d_relative_buckets(6, 5, True) if biased else (None, 0)
    leaves = [torch.tensor(x, requires_grad=True) for x in (q, k, v)]
    tt = torch.tensor(table, requires_grad=True) if biased else None
    y = torch_attention(*leaves, tt, lengths, keys, causal,
                        torch.tensor(bucket) if biased else None, rel_min)
    y.backward(torch.tensor(g))
    out, lse, _ = ref.forward(q, k, v, lengths, keys, causal, None, table, bucket, rel_min)
    grads, _, _ = ref.backward(q, k, v, g, lengths, keys, causal, None, table, bucket, rel_min)
    np.testing.assert_allclose(out, y.detach().numpy(), atol=1e-12)
    for a, b in zip(grads, leaves + ([tt] if biased else [])):
        np.testing.assert_allclose(a, b.grad.numpy(), atol=1e-11)


def test_gradients_match_differences():
    """A directional derivative of <out, g> against the gradients, with step 1e-5: the central
    difference is off by about 1e-10."""
    lengths, keys = [3, 6], [6, 4]
    q, k, v, g = inputs(3, lengths, keys, 2, 1, 4)
    table = np.random.default_rng(4).standard_normal((4, 2))
    bucket, rel_min = dsa.dsa3d_relative_buckets(4, 3, False)
    how = dict(causal=True, bucket=bucket, rel_min=rel_min)
    grads, _, _ = ref.backward(q, k, v, g, lengths, keys, table=table, **how)
    r = np.random.default_rng(5)
    for i, x in enumerate((q, k, v, table)):
        d = r.standard_normal(x.shape)
        side = []
        for e in (1e-5, -1e-5):
            y = [q, k, v, table]
            y[i] = x + e * d
            side.append((ref.forward(y[0], y[1], y[2], lengths, keys, table=y[3], **how)[0]
                         * g).sum())
        assert abs((side[0] - side[1]) / 2e-5 - (grads[i] * d).sum()) < 1e-7


def test_rows_without_keys_are_empty():
    q, k, v, g = inputs(6, [4, 2], [2, 0], 2, 2, 4)
    out, lse, _ = ref.forward(q, k, v, [4, 2], [2, 0], causal=True)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:4]).all()
    assert (out[4:] == 0).all() and np.isneginf(lse[4:]).all()
    table = np.full((2, 2), -np.inf)
    out, lse, _ = ref.forward(q, k, v, [4, 2], [2, 0], table=table, bucket=[0, 1], rel_min=0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_paged_equals_packed_where_pages_hold_the_keys():
    r = np.random.default_rng(7)
    lengths, held, size = [2, 1], [9, 5], 4
    pages = np.array([[5, 0, 2], [1, 4, -1]])
    kp, vp = r.standard_normal((2, 6, size, 2, 8))
    q = r.standard_normal((3, 4, 8))
    rows = [pages[b][j // size] * size + j % size for b, m in enumerate(held) for j in range(m)]
    k, v = kp.reshape(-1, 2, 8)[rows], vp.reshape(-1, 2, 8)[rows]
    a = ref.paged(q, kp, vp, pages, held, lengths)
    b = ref.forward(q, k, v, lengths, held, causal=True)
    for x, y in zip(a, b):
        np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("buckets,most,both", [(32, 128, True), (32, 128, False), (8, 20, True),
                                               (2, 3, False), (64, 1000, True), (256, 2047, False),
                                               (6, 5, True), (16, 64, True), (3, 1000, False)])
def test_buckets_by_whole_numbers(buckets, most, both):
    """floor((s - e) log(n / e) / log(max / e)) >= t  <=>  n^w e^t >= max^t e^w, w = s - e."""
    got, rel_min = dsa.dsa3d_relative_buckets(buckets, most, both)
    side = buckets // 2 if both else buckets
    e = side // 2
    w = side - e

    def bucket(n):
        if n < e:
            return n
        return e + max(t for t in range(w) if n ** w * e ** t >= most ** t * e ** w)

    want = [bucket(n) for n in range(most, -1, -1)]
    if both:
        want += [side + bucket(n) for n in range(1, most + 1)]
    assert got == want and rel_min == -most
