"""Which form of paged_forward_mx the calls of tests/mx_forms.py take, by the host's plan, and that
their bounds tell the roundings of alpha apart."""
import numpy as np
import pytest
import torch

from oracle import sequence as ref
from tests.mx_forms import FORMS, PRECISE, join_of, plan_query
from tests.seq_util import Bounds
from tests.test_paged_mx_rules import parts_of, plans  # noqa: F401

DIMS = (64, 128)


def test_precise_forms(plans):  # noqa: F811
    asked = [(tile, plan_query(c, D)) for tile, c in PRECISE.items() for D in DIMS]
    for (tile, _), plan in zip(asked, plans([q for _, q in asked])):
        assert plan[0] == tile and plan[1] == 1


@pytest.mark.parametrize("D", DIMS)
def test_forms(plans, D):  # noqa: F811
    asked = [plan_query(c, D) for c, _ in FORMS.values()]
    for (name, (c, form)), query, plan in zip(FORMS.items(), asked, plans(asked)):
        rows = query[0] * c.get("H", 8)
        assert (plan[0], plan[3] > 0, join_of(plan, rows)) == form, (name, plan)
        if form[2] == "8 rows":
            assert rows % 8 and 1 < plan[1] <= 64
        if form[1]:  # some of its requests are in parts, and some are not
            tiles = [-(-n * query[1] // plan[0]) for n in c["new"]]
            parts = [p for p, _ in parts_of([m if n else 0 for n, m in zip(c["new"], c["held"])],
                                            tiles, plan)]
            assert min(parts) == 1 < max(parts), (name, parts)


def bf16(x):
    return torch.tensor(x).to(torch.bfloat16).double().numpy()


def test_the_bound_tells_alphas_roundings_apart():
    """Alpha as one bf16 number breaks the bound of the calls in PRECISE, also where the result is
    divided by the sum of the rounded; as two it keeps it."""
    r = np.random.default_rng(7)
    n, m, D = 8, 40, 64
    q, k, v = (r.standard_normal((x, 1, D)) * s for x, s in ((n, 0.05), (m, 1.0), (m, 1.0)))
    o, _, mag = ref.forward(q, k, v, [n], [m], True)
    limit = Bounds("bf16", True, q, k, [n], [m], 0.0).out(o, mag)
    top = np.full((n, m), -np.inf)
    for i in range(n):
        top[i, :m - n + i + 1] = (k[:m - n + i + 1, 0] @ q[i, 0]) / 8.0
    e = np.exp(top - top.max(1, keepdims=True))
    high = bf16(e)
    both = high + bf16(e - high)
    for name, alpha, total, fits in (("plain", high, e.sum(1), False), ("own sum", high, high.sum(1),
                                     False), ("two parts", both, e.sum(1), True)):
        got = bf16(alpha @ v[:, 0] / total[:, None])
        worst = (np.abs(got - o[:, 0]) / limit[:, 0]).max()
        print(f"  {name}: {worst:.3f} of the bound")
        assert (worst <= 1.0) == fits, (name, worst)


@pytest.mark.parametrize("tile", PRECISE)
def test_every_request_has_few_keys(tile):
    assert max(PRECISE[tile]["held"]) <= 70


def test_few_requests_have_parts_for_one_round_of_workgroups(plans):  # noqa: F811
    """Up to 96 workgroups without parts: two rounds' worth of three per compute unit is slower."""
    for batch, target in ((1, 62), (4, 58), (6, 56), (7, 55), (8, 53), (12, 96), (16, 96), (64, 96)):
        plan = plans([(batch, 4, 8, batch, 30000, 128)])[0]
        assert plan[0] == 16 and plan[3] == target, (batch, plan)
