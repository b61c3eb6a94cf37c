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
