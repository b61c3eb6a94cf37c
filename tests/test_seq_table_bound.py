"""What tests/seq_table.py's tolerance sees: a table gradient computed in the roundings that are
meant passes it; one that ignores the output's residual, rounds dS to bf16 or leaves Delta's
rounding in the far buckets does not."""
import numpy as np
import pytest
import torch

from tests import seq_table

import paper_2607_22696_amd as dsa

N, H, D = 1536, 4, 64
OFFSET = 6.0  # of every value: Delta and its rounding are large beside dS


def bf16(x):
    return torch.tensor(x).bfloat16().double().numpy()


@pytest.fixture(scope="module")
def case():
    r = np.random.default_rng(5)
    q, k, v, g = (bf16(r.standard_normal((N, H, D)) * s + a)
                  for s, a in ((1.5, 0), (1, 0), (1, OFFSET), (1, 0)))
    table = r.standard_normal((6, H))
    bucket, rel_min = dsa.dsa3d_relative_buckets(6, 5, True)
    out, lse = seq_table.statistics(q, k, v, table, bucket, rel_min)
    want, limit = seq_table.table_gradient(q, k, v, g, out, lse, table, bucket, rel_min,
                                           carried=2.0 ** -18)
    return q, k, v, g, table, bucket, rel_min, out, lse, want, limit


def gradient(case, residual=True, round_ds=False, compensated=True):
    """From out as bf16 with its residual; `compensated`: pairs more than 64 from the table take
    their share of the row's sum of dS back, except in the bucket farthest behind where False."""
    q, k, v, g, table, bucket, rel_min, out, lse = case[:9]
    held = bf16(out)
    if residual:
        held = held + bf16(out - held)
    d = np.arange(N)[None, :] - np.arange(N)[:, None]
    which = np.asarray(bucket)[np.clip(d - rel_min, 0, len(bucket) - 1)]
    far = (d < rel_min - 64) | (d > rel_min + len(bucket) + 64)
    grad = np.zeros(table.shape)
    for h in range(H):
        t = q[:, h] @ k[:, h].T / np.sqrt(D) + table[which, h]
        alpha = np.exp(t - lse[:, h, None])
        ds = alpha * (g[:, h] @ v[:, h].T - (g[:, h] * held[:, h]).sum(1, keepdims=True))
        error = ds.sum(1, keepdims=True)
        if round_ds:
            ds = bf16(ds)
        take = far if compensated else far & (which != which[-1, 0])
        ds = ds - np.where(take, alpha * error, 0.0)
        for c in range(len(table)):
            grad[c, h] = ds[which == c].sum()
    return grad


def worst(case, **kw):
    want, limit = case[9:]
    return (np.abs(gradient(case, **kw) - want) / limit).max()


def test_the_meant_roundings_pass(case):
    assert worst(case) < 1.0


@pytest.mark.parametrize("how", (dict(residual=False), dict(round_ds=True),
                                 dict(compensated=False)))
def test_losses_of_precision_do_not(case, how):
    assert worst(case, **how) > 1.0


@pytest.mark.parametrize("causal", (False, True))
def test_operands_without_their_last_part(causal):
    """The spread of float32 gradients against operands of 16 bits (two bf16 parts): each result's
    root mean square error exceeds twice the root mean square of the spread, which what float32
    rounds the operands to does not."""
    r = np.random.default_rng(6)
    q, k, v, g = (r.standard_normal((300, 2, D)).astype(np.float32).astype(np.float64) * s
                  for s in (1.5, 1, 1, 1))
    want, spread = seq_table.spreads(q, k, v, g, causal)

    def short(x):
        return bf16(x) + bf16(x - bf16(x))

    for f, fits in ((short, False),
                    (lambda x: (x * (1 + 2.0 ** -24 * r.uniform(-1, 1, x.shape))), True)):
        got, _ = seq_table.spreads(*(f(x) for x in (q, k, v, g)), causal)
        for a, b, s in zip(got, want, spread):
            assert (seq_table.rms(a - b) <= 2 * seq_table.rms(s)) == fits
