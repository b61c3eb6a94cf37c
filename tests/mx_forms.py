"""Calls of paged_forward_mx that reach each of its forms, with the plan that the host makes of them
(tests/test_mx_forms.py checks that it does), for the GPU tests of those forms."""

# In few keys of about one weight each rounding of alpha shows: rows per workgroup -> call.
PRECISE = {
    16: dict(new=[1, 1, 2], held=[33, 20, 64], H=8, KH=2),
    32: dict(new=[6, 5, 7], held=[33, 20, 64], H=8, KH=2),
    128: dict(new=[60, 30, 1], held=[70, 40, 33], H=8, KH=2),
}


def plan_query(case, D):
    """(tokens, group, key heads, requests, most keys, head_dim) of a call with 16-token pages."""
    H, KH = case.get("H", 8), case.get("KH", 2)
    page = case.get("page", 16)
    columns = max([-(-m // page) for m in case["held"]] + [1]) + case.get("columns", 0)
    most = case.get("max_kv", 0)
    most = min(most, columns * page) if most else columns * page
    return (sum(case["new"]) + case.get("tail", 0), H // KH, KH, len(case["new"]), most, D)


def join_of(plan, rows):
    """Which join a call with that plan takes: none, one wave for 8 rows at a time, one for a row, or
    four for a row (csrc/paged_mx.hip, forward_d)."""
    splits = plan[1]
    if splits <= 1:
        return "none"
    if rows > 16384 and splits <= 64:
        return "8 rows"
    return "4 waves" if splits > 16 else "1 row"


def _lengths(count, most):
    """Mostly short, every 13th a long one."""
    return [most - 3 * b if b % 13 == 5 else 1 + 37 * b % 90 for b in range(count)]


# Calls of single forms: what they are, then (rows per workgroup, dealt out, join).
FORMS = {
    # requests of one part and of several beside each other, 16,407 rows: 8 at a time and 7 at the end
    "many_rows_to_join": (dict(new=[1500, 300, 20, 3], held=[3000, 300, 2500, 40], H=9, KH=9,
                               columns=20), (128, True, "8 rows")),
    "few_rows_in_few_parts": (dict(new=[1, 2, 1], held=[1400, 33, 900], H=4, KH=4, columns=60),
                              (16, True, "1 row")),
    "few_rows_in_many_parts": (dict(new=[1, 1], held=[17000, 400], H=4, KH=2),
                               (16, True, "4 waves")),
    "drafts": (dict(new=[6, 5, 0, 7, 6, 3], held=[3000, 700, 50, 65, 2100, 33]),
               (32, True, "1 row")),
    "chunks": (dict(new=[100, 3, 1, 40], held=[4000, 700, 2600, 41], H=4, KH=1),
               (128, True, "1 row")),
    "66_drafts": (dict(new=[6, 8] * 33, held=_lengths(66, 1500)), (32, False, "1 row")),
    "66_tokens": (dict(new=[1] * 66, held=_lengths(66, 1500)), (16, False, "1 row")),
    "66_chunks": (dict(new=[30] * 66, held=_lengths(66, 1500), H=4, KH=1), (128, False, "1 row")),
}
