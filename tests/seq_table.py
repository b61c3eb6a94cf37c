"""The table gradient of a relative position bias from given statistics, in float64, and how far
float32 arithmetic may take it.

tests/seq_util.py bounds a sum by the absolute values of its terms, which for a sum of millions of
terms of either sign says little.  Here the roundings of different rows and pairs count as
independent, so that their squares add, and a result may be off by four standard deviations:

  (a rounding of x to float32 is off by 2^-25 |x| in the mean, one of the matrix cores, which
  do not round to nearest, by 2^-24)
  a row's weights have one relative error, of lse, of lse log2(e) and of the logarithm and the
      product that lse came from:     e_row = (3 |lse| + 4) 2^-25
  a pair's own: the logit's (float32 sum of D products in D / 16 steps), the exponent's and the
      exponential's, the dot product dP's:
      e_pair = (|t - lse| + 2 (|t| + 1) sqrt(D / 16) + 4) 2^-25
  a row's Delta = <dout, O>, in units of |dout O| = sqrt(sum dout^2 O^2): float32 sums of D terms
      and of the row's dS (m / 32 blocks), (sqrt(D) + sqrt(m / 32)) 2^-25, and what O is off,
      `carried`: where out and out_res hold it, the residual's rounding is 2^-18.7 of a channel in
      the mean over a binade, the rounding of the weights' two parts the same again, 2^-18
      together.  The row's own sum of dS, zero where the statistics are of its own keys alone,
      tells that part, and it stays only in the 32 x 32 blocks that reach into the table: pairs
      less than 64 from it.
"""
import numpy as np

from oracle import sequence as ref

SIGMAS = 4.0


def table_gradient(q, k, v, dout, out, lse, table, bucket, rel_min, causal=False, carried=0.0,
                   shift=0):
    """d_table [buckets, heads] of one sequence whose weights are exp(t - lse) and whose Delta is
    <dout, out>, and its tolerance.  `shift` is added to the distances (the keys' place among
    more)."""
    n, m, H, D = len(q), len(k), q.shape[1], q.shape[2]
    grad, var = np.zeros(table.shape), np.zeros(table.shape)
    d = np.arange(m)[None, :] - (np.arange(n)[:, None] + m - n)
    which = np.asarray(bucket)[np.clip(d + shift - rel_min, 0, len(bucket) - 1)]
    inside = (d + shift > rel_min - 64) & (d + shift < rel_min + len(bucket) + 64)
    sums = (np.sqrt(D) + np.sqrt(m / 32)) * 2.0 ** -25
    for h in range(H):
        u = h // (H // k.shape[1])
        t = q[:, h] @ k[:, u].T / np.sqrt(D) + table[which, h]
        alpha = np.exp(t - lse[:, h, None])
        if causal:
            alpha = np.where(d > 0, 0.0, alpha)
        dp = dout[:, h] @ v[:, u].T
        delta = (dout[:, h] * out[:, h]).sum(1, keepdims=True)
        unit = np.sqrt((dout[:, h] ** 2 * out[:, h] ** 2).sum(1))
        ds = alpha * (dp - delta)
        e_row = (3 * np.abs(lse[:, h]) + 4) * 2.0 ** -25
        e_pair = (np.abs(t - lse[:, h, None]) + 2 * (np.abs(t) + 1) * np.sqrt(D / 16) + 4)
        e_pair = e_pair * 2.0 ** -25
        pair = (alpha * (np.abs(dp) + np.abs(delta)) * e_pair) ** 2
        for c in range(len(table)):
            at = which == c
            grad[c, h] = ds[at].sum()
            row = (np.where(at, ds, 0.0).sum(1) * e_row) ** 2
            summed = (np.where(at, alpha, 0.0).sum(1) * unit * sums) ** 2
            near = (np.where(at & inside, alpha, 0.0).sum(1) * unit * carried) ** 2
            var[c, h] = pair[at].sum() + (row + summed + near).sum()
    return grad, SIGMAS * np.sqrt(var) + 1e-30


def statistics(q, k, v, table, bucket, rel_min, causal=False):
    """out and lse of one sequence in float64."""
    return ref.forward(q, k, v, [len(q)], [len(k)], causal, None, table, bucket, rel_min)[:2]


def spreads(q, k, v, dout, causal=False):
    """out, dq, dk, dv of one sequence in float64 and the standard deviations that float32
    roundings give their elements: each pair's weight by e_row and e_pair, its dS by |dP| +
    |Delta| times these."""
    n, m, H, D = len(q), len(k), q.shape[1], q.shape[2]
    out, lse, _ = ref.forward(q, k, v, [n], [m], causal)
    grads = ref.backward(q, k, v, dout, [n], [m], causal)[0][:3]
    values = (out, *grads)
    var = [np.zeros(x.shape) for x in values]
    for h in range(H):
        u = h // (H // k.shape[1])
        t = q[:, h] @ k[:, u].T / np.sqrt(D)
        alpha = np.exp(t - lse[:, h, None])
        if causal:
            alpha = np.where(np.arange(m)[None, :] > np.arange(n)[:, None] + (m - n), 0.0, alpha)
        e2 = ((3 * np.abs(lse[:, h, None]) + 4) * 2.0 ** -25) ** 2 + \
            ((np.abs(t - lse[:, h, None]) + 2 * (np.abs(t) + 1) * np.sqrt(D / 16) + 4)
             * 2.0 ** -25) ** 2
        size = alpha * (np.abs(dout[:, h] @ v[:, u].T) +
                        np.abs((dout[:, h] * out[:, h]).sum(1, keepdims=True)))
        a2, s2 = alpha ** 2 * e2, size ** 2 * e2 / D
        var[0][:, h] += a2 @ v[:, u] ** 2
        var[1][:, h] += s2 @ k[:, u] ** 2
        var[2][:, u] += s2.T @ q[:, h] ** 2
        var[3][:, u] += a2.T @ dout[:, h] ** 2
    return values, [np.sqrt(x) for x in var]


def rms(x):
    return float(np.sqrt((x ** 2).mean()))
