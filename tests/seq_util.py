"""Inputs and error bounds of the sequence tests.

Bounds, from the kernels' roundings (u = half a unit in the last place of the storage type: bf16
2^-8, float32 2^-24; e = 2^-23 for one float32 operation, the matrix cores not rounding to
nearest):
  a logit is a float32 sum of D exact products times the scale, plus a bias:
      dt = e ((D + 4) scale max sum |q| |k| + 4 max |table|), relative error of alpha 2 dt + m e
  out = sum alpha v: alpha rounded to the operand type (half: bf16 2^-8, 2^-17 with a residual,
      float32 none), summed in float32, rounded once to storage.
  dS = alpha (dP - Delta): the relative error of alpha, D e of the two dot products, the operand
      rounding, and alpha times |dout| times what the read `out` is off.
Every bound is a sum of absolute values of terms (the oracle's magnitudes) times these.
"""
import numpy as np
import torch

from oracle import sequence as ref

E32 = 2.0 ** -23
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
UNIT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def rounded(r, shape, dtype, std=1.0):
    """Normal numbers as the storage type has them: a CPU tensor and its float64 values."""
    t = torch.tensor(r.standard_normal(shape) * std).to(TYPES[dtype])
    return t, t.double().numpy()


class Bounds:
    def __init__(self, dtype, residual, q, k, lengths, keys, scale, table=None):
        D, group = q.shape[2], q.shape[1] // max(k.shape[1], 1)
        top, self.m = 0.0, max([1] + list(keys))
        self.n = max([1] + list(lengths)) * group
        cq, ck = ref.starts(lengths), ref.starts(keys)
        for b, (n, m) in enumerate(zip(lengths, keys)):
            if n and m:
                for h in range(q.shape[1]):
                    a = np.abs(q[cq[b]:cq[b] + n, h]) @ np.abs(k[ck[b]:ck[b] + m, h // group]).T
                    top = max(top, float(a.max()))
        big = 0.0
        if table is not None:
            kept = table[table > ref.HIDDEN]
            big = float(np.abs(kept).max()) if kept.size else 0.0
        scale = scale or D ** -0.5
        self.dt = E32 * ((D + 4) * scale * top + 4 * big)
        self.alpha = 2 * self.dt + self.m * E32 + 4 * E32
        self.operand = {"f32": 0.0, "bf16": 2.0 ** -8}[dtype]
        self.out_operand = 2.0 ** -17 if residual else self.operand
        self.unit, self.D, self.residual = UNIT[dtype], D, residual

    def out(self, out, mag):
        return mag * (self.alpha + self.out_operand + self.m * E32) + np.abs(out) * self.unit

    def read_out(self, out, mag):
        unit = 2.0 ** -16 if self.residual else self.unit
        return mag * (self.alpha + self.out_operand + self.m * E32) + np.abs(out) * unit

    def lse(self, lse):
        return 2 * self.dt + self.m * E32 + np.abs(np.where(np.isfinite(lse), lse, 0)) * 4 * E32

    def grads(self, grads, mags, extra):
        sums = (self.m, self.n, self.n, self.m * self.n)
        res = []
        for i, (g, mag, ex, terms) in enumerate(zip(grads, mags, extra, sums)):
            rel = self.alpha + 2 * self.D * E32 + min(terms, 4096) * E32
            if i < 3:
                rel += self.operand
            res.append(mag * rel + ex * (1 + rel) + np.abs(g) * (self.unit if i < 3 else E32))
        return res


def near(name, got, want, bound):
    got = got.detach().double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    whole = np.isfinite(want)
    assert np.array_equal(got[~whole], want[~whole], equal_nan=True), name
    off = np.abs(got[whole] - want[whole])
    limit = (bound + np.zeros_like(want))[whole] + 1e-30
    worst = float((off / limit).max()) if off.size else 0.0
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    assert np.isfinite(got[whole]).all() and worst <= 1.0, (name, worst)
