"""Plain attention of packed sequences and over a paged cache in float64, head by head, written
from the formulas of include/dsa3d_seq.h; used by the tests only.

Beside each result stands what the rounding of the kernels can make of it: `mag` holds the sums
of the absolute values of the terms, from which `bounds` derives how far float32 arithmetic with
bf16 operands may be off.
"""
from __future__ import annotations

import numpy as np

HIDDEN = -1e30  # a bias at or below this hides its keys


def starts(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def bias_matrix(n, m, column, bucket, rel_min):
    """[n, m] of column[bucket[clamped distance]], 0 where the bucket is none of the column's."""
    d = np.arange(m)[None, :] - (np.arange(n)[:, None] + m - n)
    b = np.asarray(bucket)[np.clip(d - rel_min, 0, len(bucket) - 1)]
    ok = (b >= 0) & (b < len(column))
    return np.where(ok, column[np.where(ok, b, 0)], 0.0), np.where(ok, b, -1)


def weights(q, k, causal, scale, bias, there=None):
    """alpha [n, m] and lse [n] of one head; `there`: keys that exist.  A row without keys has
    alpha 0 and lse -inf."""
    n, m = len(q), len(k)
    seen = np.ones((n, m), bool)
    if causal:
        seen &= np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)
    if there is not None:
        seen &= there[None, :]
    if bias is not None:
        seen &= ~(bias <= HIDDEN)
    k = np.where(seen.any(0)[:, None], k, 0.0)
    t = (q @ k.T) * scale + (0.0 if bias is None else np.where(seen, bias, 0.0))
    t = np.where(seen, t, -np.inf)
    top = t.max(1, initial=-np.inf)
    e = np.exp(t - np.where(np.isfinite(top), top, 0.0)[:, None])
    total = e.sum(1)
    some = total > 0
    lse = np.full(n, -np.inf)
    lse[some] = top[some] + np.log(total[some])
    return np.where(seen, e / np.where(some, total, 1.0)[:, None], 0.0), lse, seen


def forward(q, k, v, lengths, keys, causal=False, scale=None, table=None, bucket=None, rel_min=0):
    """out, lse and mag (the sums of alpha |v|); rows behind the last sequence: 0 and -inf."""
    H, KH, D = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or 1.0 / np.sqrt(D)
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    cq, ck = starts(lengths), starts(keys)
    for b, (n, m) in enumerate(zip(lengths, keys)):
        qs, ks = slice(cq[b], cq[b] + n), slice(ck[b], ck[b] + m)
        for h in range(H):
            u = h // (H // KH)
            bias = None if table is None else bias_matrix(n, m, table[:, h], bucket, rel_min)[0]
            a, lse[qs, h], _ = weights(q[qs, h], k[ks, u], causal, scale, bias)
            out[qs, h], mag[qs, h] = a @ v[ks, u], a @ np.abs(v[ks, u])
    return out, lse, mag


def backward(q, k, v, dout, lengths, keys, causal=False, scale=None, table=None, bucket=None,
             rel_min=0, out_error=None):
    """dq, dk, dv, d_table, and their magnitudes in the same order: the sums of |terms| in which
    every dS counts |dS| `plus` alpha times the error that Delta takes from out_error (how far
    out, as the backward reads it, may be off)."""
    H, KH, D = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or 1.0 / np.sqrt(D)
    grads = [np.zeros(x.shape) for x in (q, k, v)]
    mags = [np.zeros(x.shape) for x in (q, k, v)]
    extra = [np.zeros(x.shape) for x in (q, k, v)]
    dt, mt, et = (np.zeros((1, H) if table is None else table.shape) for _ in range(3))
    cq, ck = starts(lengths), starts(keys)
    for b, (n, m) in enumerate(zip(lengths, keys)):
        qs, ks = slice(cq[b], cq[b] + n), slice(ck[b], ck[b] + m)
        for h in range(H):
            u = h // (H // KH)
            bias = which = None
            if table is not None:
                bias, which = bias_matrix(n, m, table[:, h], bucket, rel_min)
            x, y, z, g = q[qs, h], k[ks, u], v[ks, u], dout[qs, h]
            a, _, seen = weights(x, y, causal, scale, bias)
            some = seen.any(1)
            g = np.where(some[:, None], g, 0.0)
            dp = g @ z.T
            ds = a * (dp - (a * dp).sum(1, keepdims=True))
            off = 0.0 if out_error is None else \
                a * (np.abs(g) * out_error[qs, h]).sum(1, keepdims=True)
            size = a * (np.abs(g) @ np.abs(z).T + (np.abs(g) * np.abs(a @ z)).sum(1, keepdims=True))
            for i, (at, hd, left) in enumerate(((qs, h, False), (ks, u, True))):
                other = x if left else y
                for store, d, r in ((grads, ds, other), (mags, size, np.abs(other)),
                                    (extra, off, np.abs(other))):
                    if isinstance(d, float):
                        continue
                    store[i][at, hd] += scale * ((d.T if left else d) @ r)
            grads[2][ks, u] += a.T @ g
            mags[2][ks, u] += a.T @ np.abs(g)
            if table is not None:
                for c in range(len(table)):
                    at = which == c
                    dt[c, h] += ds[at].sum()
                    mt[c, h] += size[at].sum()
                    et[c, h] += 0.0 if isinstance(off, float) else off[at].sum()
    return (*grads, dt), (*mags, mt), (*extra, et)


def gather(k_pages, v_pages, row, held):
    """Tokens 0 .. held - 1 of a request, and which of them have a page."""
    size, num = k_pages.shape[1], k_pages.shape[0]
    at = np.arange(held)
    page = np.asarray(row)[at // size] if held else np.zeros(0, int)
    there = (page >= 0) & (page < num)
    page = np.where(there, page, 0)
    zero = lambda x: np.where(there[:, None, None], x[page, at % size], 0.0)  # noqa: E731
    return zero(k_pages), zero(v_pages), there


def paged(q, k_pages, v_pages, pages, held, lengths, causal=True, scale=None, table=None,
          bucket=None, rel_min=0):
    """out, lse, mag of new tokens over their requests' pages."""
    H, D = q.shape[1], q.shape[2]
    scale = scale or 1.0 / np.sqrt(D)
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    cq = starts(lengths)
    for b, (n, m) in enumerate(zip(lengths, held)):
        k, v, there = gather(k_pages, v_pages, pages[b], m)
        qs = slice(cq[b], cq[b] + n)
        for h in range(H):
            u = h // (H // k.shape[1])
            bias = None if table is None else bias_matrix(n, m, table[:, h], bucket, rel_min)[0]
            a, lse[qs, h], _ = weights(q[qs, h], k[:, u], causal, scale, bias, there)
            out[qs, h], mag[qs, h] = a @ v[:, u], a @ np.abs(v[:, u])
    return out, lse, mag


def append(k, v, k_pages, v_pages, pages, held, lengths):
    """The pages with each new token written to its place, tokens without one dropped."""
    k_pages, v_pages = k_pages.copy(), v_pages.copy()
    num, size = k_pages.shape[:2]
    at = 0
    for b, (n, m) in enumerate(zip(lengths, held)):
        for i in range(n):
            j = m - n + i
            if 0 <= j < pages.shape[1] * size and 0 <= pages[b, j // size] < num:
                k_pages[pages[b, j // size], j % size] = k[at + i]
                v_pages[pages[b, j // size], j % size] = v[at + i]
        at += n
    return k_pages, v_pages
