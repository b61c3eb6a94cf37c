"""Performance cases of the sequence operators: attention of packed sequences, with a learned
relative position bias, and over a paged cache.

Video tokens stand on a grid; the prompts that condition them, and the tokens that a language
model writes for them, are sequences of different lengths.  Four operators, each in the form
that a program which holds its tensors on the GPU runs:

  `seq`     softmax attention of packed sequences, causal or not, queries in groups that share a
            key head, keys of the same or of other sequences; a forward or a training step
  `bias`    the same with a learned bias of the relative position, one value per bucket of
            distances and head, and the table's gradient
  `paged`   attention of the newest tokens of each request over keys and values kept in pages
  `append`  the keys and values of the newest tokens written into those pages

With `own` false every pass is computed in elementary torch operations in 32 bits (64 for the
sums over whole diagonals), rounded once; with `own` true it makes the library's calls.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ITEM = {"bf16": 2, "f32": 4}
_BUCKETS, _MAX_DISTANCE = 32, 128


# ----------------------------------------------------------------------------- cases

def _seq(name, kind, lengths, heads, kv_heads, head_dim, dtype, causal, keys="", op="seq"):
    """`lengths`, `keys`: tokens of each sequence, separated by spaces; no `keys`: the same."""
    return {"name": name, "op": op, "pass": kind, "lengths": lengths, "keys": keys,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype,
            "causal": causal}


def _paged(name, op, new, held, heads, kv_heads, head_dim, page, dtype, bias=False):
    """`new`: tokens of each request in this call; `held`: all its tokens, those included."""
    return {"name": name, "op": op, "new": new, "held": held, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype,
            "bias": bias}


def _text(numbers):
    return " ".join(str(n) for n in numbers)


def _spread(count, lo, hi):
    """`count` lengths between lo and hi, uneven and in no order."""
    return [lo + (hi - lo) * ((7 * i + 3) % count) // max(count - 1, 1) for i in range(count)]


def listed():
    return [
        # the smallest call: a handful of short prompts, where launches and host work are the time
        _seq("seq_fwd_short_prompts", "forward", "1 37 5 64 20", 16, 16, 64, "bf16", False),
        # cross-attention of two clips' video tokens (two frames of the 68 x 120 grid, four of
        # the 34 x 60 grid) to their prompts, 24 heads x 128
        _seq("seq_fwd_cross_prompts", "forward", "16320 8160", 24, 24, 128, "bf16", False,
             keys="226 77"),
        # reading a long document: one causal sequence
        _seq("seq_fwd_causal_16k", "forward", "16384", 16, 4, 128, "bf16", True),
        # training a decoder on packed documents of different lengths, grouped heads
        _seq("seq_step_causal_packed", "step", "4096 517 1333 2246", 32, 8, 128, "bf16", True),
        # a small model trained in fp32 on odd lengths
        _seq("seq_step_f32_odd", "step", "100 1 333 257 1030", 6, 2, 64, "f32", True),
        # a text encoder over a batch of prompts, biased by the distance in both directions
        _seq("bias_fwd_encoder", "forward", _text(_spread(24, 40, 512)), 24, 24, 64, "bf16",
             False, op="bias"),
        # the same encoder trained on longer texts, with the table's gradient
        _seq("bias_step_encoder", "step", "1024 700 2048 311 13", 16, 16, 64, "bf16", False,
             op="bias"),
        # writing one token for one user: the shortest serving step
        _paged("paged_one_request", "paged", "1", "700", 32, 8, 128, 16, "bf16"),
        # writing one token each for 64 users whose caches differ in length
        _paged("paged_decode_64", "paged", _text([1] * 64), _text(_spread(64, 200, 8000)), 32, 8,
               128, 16, "bf16"),
        # reading prompts in chunks beside users that are being written to, long caches
        _paged("paged_chunks", "paged", "512 1 801 1 1 300", "16000 3001 801 77 9000 5000", 32, 8,
               128, 64, "bf16"),
        # the cache's side of a writing step
        _paged("append_decode_64", "append", _text([1] * 64), _text(_spread(64, 20, 500)), 32, 8,
               128, 16, "bf16"),
        # the cache's side of reading prompts
        _paged("append_prompts", "append", "4096 1000 2500 1", "4096 1500 6000 900", 32, 8, 128,
               64, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((1, 1), (6, 6), (16, 16), (8, 2), (12, 4), (32, 8), (24, 24), (16, 1))


def draw(rng):
    op = rng.choice(("seq", "seq", "bias", "paged", "paged", "append"))
    heads, kv_heads = rng.choice(_HEADS)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    head_dim = rng.choice((64, 128))
    if op in ("seq", "bias"):
        kind = rng.choice(("forward", "step"))
        causal = rng.random() < 0.6
        count = _log_int(rng, 1, 24)
        lengths = [_log_int(rng, 1, 6000) for _ in range(count)]
        keys = []
        if op == "seq" and rng.random() < 0.25:
            causal, keys = False, [_log_int(rng, 1, 600) for _ in range(count)]
        # at most the pairs of the largest listed case of each direction, padding included
        most = 16384 * 16384 * 16 // (2 if kind == "forward" else 6)
        while _padded(lengths, keys) * heads * (2 if dtype == "f32" else 1) > most:
            longest = lengths.index(max(lengths))
            lengths[longest] = max(1, lengths[longest] * 2 // 3)
            if len(lengths) > 1 and max(lengths) < 3 * sum(lengths) // len(lengths):
                lengths.pop()
                keys = keys[:-1]
        case = _seq("", kind, _text(lengths), heads, kv_heads, head_dim, dtype, causal,
                    _text(keys), op)
        del case["name"]
        return case
    count = _log_int(rng, 1, 64)
    chunk = rng.choice((1, 1, 4, 900))
    new = [_log_int(rng, 1, chunk) for _ in range(count)]
    held = [n + _log_int(rng, 1, 8000) for n in new]
    rows = 6000 if op == "paged" else 60000
    while sum(held) * kv_heads > 2000 * rows or \
            len(new) * max(new) * max(held) * heads > 16384 ** 2 * 8:
        drop = held.index(max(held))
        del held[drop], new[drop]
        if not held:
            held, new = [300], [1]
    page = rng.choice((16, 16, 32, 64, 128))
    if op == "append":
        held = [n + (h - n) // 8 for n, h in zip(new, held)]
    case = _paged("", op, _text(new), _text(held), heads, kv_heads, head_dim, page, dtype,
                  op == "paged" and rng.random() < 0.3)
    del case["name"]
    return case


def _padded(lengths, keys):
    return len(lengths) * max(lengths) * max(keys or lengths)


# ----------------------------------------------------------------------------- inputs

def _numbers(text):
    return [int(n) for n in text.split()]


def _starts(lengths):
    total = [0]
    for n in lengths:
        total.append(total[-1] + n)
    return total


def _bucket_map(both):
    """Buckets of the distances key - query from -128 to 128 (to 0 where keys ahead are hidden):
    half of them exact, the rest widening with the logarithm up to the last, which takes all
    farther ones.  Whole-number arithmetic, so that a distance at a border falls to its side."""
    side = _BUCKETS // 2 if both else _BUCKETS
    exact_to = side // 2
    wide = side - exact_to

    def bucket(n):
        if n < exact_to:
            return n
        t = 0
        while t + 1 < wide and (n ** wide) * exact_to ** (t + 1) >= \
                (_MAX_DISTANCE ** (t + 1)) * exact_to ** wide:
            t += 1
        return exact_to + t

    behind = [bucket(n) for n in range(_MAX_DISTANCE, -1, -1)]
    ahead = [side + bucket(n) for n in range(1, _MAX_DISTANCE + 1)] if both else []
    return behind + ahead


def _normal(gen, shape, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, D = _TYPES[case["dtype"]], case["head_dim"]
    H, G = case["heads"], case["kv_heads"]
    state = {"case": case, "scale": 1.0 / math.sqrt(D)}
    # queries a little longer than unit length give rows with some keys that stand out
    if case["op"] in ("seq", "bias"):
        lengths = _numbers(case["lengths"])
        keys = _numbers(case["keys"]) or lengths
        nq, nk = sum(lengths), sum(keys)
        state.update(lengths=lengths, keys=keys, cu_q=_ints(_starts(lengths)),
                     cu_k=_ints(_starts(keys)) if case["keys"] else None,
                     q=_normal(gen, (nq, H, D), dt, 1.5), k=_normal(gen, (nk, G, D), dt),
                     v=_normal(gen, (nk, G, D), dt))
        if case["pass"] == "step":
            state["dout"] = _normal(gen, (nq, H, D), dt)
        biased = case["op"] == "bias"
    else:
        new, held, page = _numbers(case["new"]), _numbers(case["held"]), case["page"]
        nq = sum(new)
        counts = [-(-n // page) for n in held]
        # pages are handed out as requests grow, so that a request's pages lie scattered
        order = torch.randperm(sum(counts), generator=gen, device="cuda").to(torch.int32).cpu()
        table = torch.full((len(held), max(counts)), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(counts):
            table[b, :c] = order[at:at + c]
            at += c
        state.update(lengths=new, keys=held, page=page, cu_q=_ints(_starts(new)),
                     kv_lens=_ints(held), table=table.cuda(),
                     k_pages=_normal(gen, (sum(counts), page, G, D), dt),
                     v_pages=_normal(gen, (sum(counts), page, G, D), dt))
        if case["op"] == "paged":
            state["q"] = _normal(gen, (nq, H, D), dt, 1.5)
        else:
            state.update(k=_normal(gen, (nq, G, D), dt), v=_normal(gen, (nq, G, D), dt))
        biased = case["bias"]
    if biased:
        both = not case.get("causal", True)
        state.update(rel_buckets=_ints(_bucket_map(both)), rel_min=-_MAX_DISTANCE,
                     rel_table=_normal(gen, (_BUCKETS, H), torch.float32))
    return state


# ----------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    if op in ("seq", "bias"):
        return _plain_attention(state)
    return _plain_paged(state) if op == "paged" else _plain_append(state)


def _own_attention(s):
    import paper_2607_22696_amd as dsa
    case = s["case"]
    how = dict(cu_k=s["cu_k"], causal=case["causal"], scale=s["scale"])
    if case["op"] == "bias":
        how.update(rel_table=s["rel_table"], rel_buckets=s["rel_buckets"], rel_min=s["rel_min"])
    step = case["pass"] == "step"
    out, lse, res = dsa.seq_forward(s["q"], s["k"], s["v"], s["cu_q"], need_lse=step,
                                    need_residual=step and case["op"] == "bias", **how)
    if not step:
        return {"out": out}
    grads = dsa.seq_backward(s["q"], s["k"], s["v"], out, res, lse, s["dout"], s["cu_q"], **how)
    return {"out": out, "lse": lse,
            **dict(zip(("dq", "dk", "dv", "d_rel_table"), grads))}


def _own_paged(s):
    import paper_2607_22696_amd as dsa
    how = {}
    if s["case"]["bias"]:
        how.update(rel_table=s["rel_table"], rel_buckets=s["rel_buckets"], rel_min=s["rel_min"])
    out, _ = dsa.paged_forward(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_lens"],
                               s["cu_q"], scale=s["scale"], max_kv=max(s["keys"]), **how)
    return {"out": out}


def _own_append(s):
    import paper_2607_22696_amd as dsa
    dsa.paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["kv_lens"],
                     s["cu_q"])
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


_OWN = {"seq": _own_attention, "bias": _own_attention, "paged": _own_paged,
        "append": _own_append}


def _rows(starts, counts, width):
    """Rows of a packed tensor as [sequence, width], and which of them are a sequence's own."""
    at = torch.arange(width, device="cuda")
    there = at < counts[:, None]
    return torch.where(there, starts[:, None] + at, 0).long(), there


def _take(x, rows, there, groups=1):
    """[rows, heads, D] as [sequence, heads x groups, width, D] in 32 bits, zeros elsewhere."""
    y = torch.where(there[..., None, None], x[rows].float(), 0.0).transpose(1, 2)
    return y.repeat_interleave(groups, dim=1).contiguous()


def _hidden(there_q, there_k, ahead, causal):
    """Pairs [sequence, 1, query, key] that no sum takes; `ahead`: key - query position."""
    hide = ~(there_q[:, :, None] & there_k[:, None, :])
    if causal:
        hide = hide | (ahead > 0)
    return hide[:, None]


def _softmax(logits):
    """Weights and log-sum-exp of each row; a row with no key has neither."""
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    weights = torch.exp(logits - top)
    total = weights.sum(-1, keepdim=True)
    weights = torch.where(total > 0, weights / total, 0.0)
    return weights, (top + torch.log(total))[..., 0]


def _bias_of(s, ahead):
    """The bias [sequence, heads, query, key] of the distances `ahead`."""
    last = s["rel_buckets"].numel() - 1
    at = s["rel_buckets"][(ahead - s["rel_min"]).clamp(0, last)].long()
    return s["rel_table"][at].permute(0, 3, 1, 2)


def _pack(x, rows, there, like):
    """[sequence, heads, width, D] back to rows, rounded to the type of `like`."""
    y = torch.zeros(like.shape, dtype=like.dtype, device="cuda")
    y[rows[there]] = x.transpose(1, 2)[there].to(like.dtype)
    return y


def _plain_attention(s):
    case = s["case"]
    groups = case["heads"] // case["kv_heads"]
    cq, ck = s["cu_q"], s["cu_q"] if s["cu_k"] is None else s["cu_k"]
    nq, nk = cq.diff(), ck.diff()
    qr, qt = _rows(cq[:-1], nq, max(s["lengths"]))
    kr, kt = _rows(ck[:-1], nk, max(s["keys"]))
    q, k, v = _take(s["q"], qr, qt), _take(s["k"], kr, kt, groups), _take(s["v"], kr, kt, groups)
    pos = torch.arange(qr.shape[1], device="cuda") + (nk - nq)[:, None]
    ahead = torch.arange(kr.shape[1], device="cuda") - pos[:, :, None]
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if case["op"] == "bias":
        logits += _bias_of(s, ahead)
    logits.masked_fill_(_hidden(qt, kt, ahead, case["causal"]), -math.inf)
    p, lse = _softmax(logits)
    del logits
    result = {"out": _pack(torch.matmul(p, v), qr, qt, s["q"])}
    if case["pass"] == "forward":
        return result
    result["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    result["lse"][qr[qt]] = lse.transpose(1, 2)[qt]
    g = _take(s["dout"], qr, qt)
    ds = torch.matmul(g, v.transpose(2, 3).contiguous())
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p)
    summed = lambda x: x.unflatten(1, (case["kv_heads"], groups)).sum(2)  # noqa: E731
    result["dq"] = _pack(torch.matmul(ds, k) * s["scale"], qr, qt, s["q"])
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * s["scale"]
    result["dk"] = _pack(summed(dk), kr, kt, s["k"])
    result["dv"] = _pack(summed(torch.matmul(p.transpose(2, 3).contiguous(), g)), kr, kt, s["v"])
    if case["op"] == "bias":
        result["d_rel_table"] = _table_gradient(s, ds)
    return result


def _table_gradient(s, ds):
    """Sums of ds over the pairs of each bucket: first over each diagonal, which a row-by-row
    shift turns into a column, in 64 bits."""
    n = ds.shape[-1]
    flat = torch.nn.functional.pad(ds.sum(0, dtype=torch.float64).flip(1), (0, n)).flatten(1)
    diagonals = flat[:, :n * (2 * n - 1)].unflatten(1, (n, 2 * n - 1)).sum(1)
    ahead = torch.arange(1 - n, n, device="cuda")
    at = s["rel_buckets"][(ahead - s["rel_min"]).clamp(0, s["rel_buckets"].numel() - 1)]
    which = (at == torch.arange(_BUCKETS, device="cuda")[:, None]).double()
    return torch.matmul(which, diagonals.transpose(0, 1).contiguous()).float()


def _slots(s, width):
    """Where tokens 0 .. width - 1 of each request lie in the flattened pages."""
    at = torch.arange(width, device="cuda")
    pages = s["table"][:, at // s["page"]].long()
    return (pages * s["page"] + at % s["page"]).clamp_min(0)


def _plain_paged(s):
    case = s["case"]
    groups = case["heads"] // case["kv_heads"]
    new = s["cu_q"].diff()
    qr, qt = _rows(s["cu_q"][:-1], new, max(s["lengths"]))
    kr, kt = _slots(s, max(s["keys"])), \
        torch.arange(max(s["keys"]), device="cuda") < s["kv_lens"][:, None]
    q = _take(s["q"], qr, qt)
    k = _take(s["k_pages"].flatten(0, 1), kr, kt, groups)
    v = _take(s["v_pages"].flatten(0, 1), kr, kt, groups)
    pos = torch.arange(qr.shape[1], device="cuda") + (s["kv_lens"] - new)[:, None]
    ahead = torch.arange(kr.shape[1], device="cuda") - pos[:, :, None]
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if case["bias"]:
        logits += _bias_of(s, ahead)
    logits.masked_fill_(_hidden(qt, kt, ahead, True), -math.inf)
    return {"out": _pack(torch.matmul(_softmax(logits)[0], v), qr, qt, s["q"])}


def _plain_append(s):
    new = s["cu_q"].diff()
    qr, qt = _rows(s["cu_q"][:-1], new, max(s["lengths"]))
    pos = torch.arange(qr.shape[1], device="cuda") + (s["kv_lens"] - new)[:, None]
    pages = s["table"].gather(1, torch.where(qt, pos // s["page"], 0).long()).long()
    at = (pages * s["page"] + pos % s["page"])[qt]
    s["k_pages"].flatten(0, 1)[at] = s["k"][qr[qt]]
    s["v_pages"].flatten(0, 1)[at] = s["v"][qr[qt]]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ----------------------------------------------------------------------------- work

def _pairs(queries, keys, causal):
    """Query-key pairs that the mask leaves: query i of n sees m - n + i + 1 of m keys."""
    if not causal:
        return sum(n * m for n, m in zip(queries, keys))
    return sum(sum(max(0, m - n + i + 1) for i in range(n)) for n, m in zip(queries, keys))


def work(case):
    item, H, G, D = _ITEM[case["dtype"]], case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] in ("seq", "bias"):
        lengths = _numbers(case["lengths"])
        keys = _numbers(case["keys"]) or lengths
        q, kv = sum(lengths) * H * D * item, 2 * sum(keys) * G * D * item
        pairs = _pairs(lengths, keys, case["causal"]) * H * D
        if case["pass"] == "forward":
            return {"bytes": 2 * q + kv, "flops": 4 * pairs}
        # forward and backward: q, k, v, dout in; out, lse, dq, dk, dv out
        return {"bytes": 4 * q + 2 * kv + 4 * sum(lengths) * H, "flops": 14 * pairs}
    new, held = _numbers(case["new"]), _numbers(case["held"])
    if case["op"] == "append":
        return {"bytes": 4 * sum(new) * G * D * item, "flops": 0}
    return {"bytes": 2 * sum(new) * H * D * item + 2 * sum(held) * G * D * item,
            "flops": 4 * _pairs(new, held, True) * H * D}


# ----------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """Sequence by sequence and head by head in float64, gradients by differentiation."""
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    heads, groups = case["heads"], case["heads"] // case["kv_heads"]
    paged = case["op"] == "paged"
    step = not paged and case["pass"] == "step"
    causal = True if paged else case["causal"]
    biased = case["bias"] if paged else case["op"] == "bias"
    if paged:
        table = s["table"].tolist()
        held = [[table[b][t // s["page"]] * s["page"] + t % s["page"] for t in range(n)]
                for b, n in enumerate(s["keys"])]
        rows = torch.tensor([r for h in held for r in h], device="cuda")
        k, v = (s[n].flatten(0, 1)[rows].double() for n in ("k_pages", "v_pages"))
    else:
        k, v = s["k"].double(), s["v"].double()
    q = s["q"].double()
    leaves = [q, k, v]
    table = s["rel_table"].double() if biased else None
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    grads = [torch.zeros_like(x) for x in leaves + ([table] if biased else [])]
    q0 = k0 = 0
    for n, m in zip(s["lengths"], s["keys"]):
        i = torch.arange(n, device="cuda")[:, None] + (m - n)
        j = torch.arange(m, device="cuda")[None, :]
        bucket = None
        if biased:
            clamped = (j - i).clamp(s["rel_min"], s["rel_min"] + s["rel_buckets"].numel() - 1)
            bucket = s["rel_buckets"].long()[clamped - s["rel_min"]]
        for h in range(heads):
            a = q[q0:q0 + n, h].clone().requires_grad_(step)
            b = k[k0:k0 + m, h // groups].clone().requires_grad_(step)
            c = v[k0:k0 + m, h // groups].clone().requires_grad_(step)
            t = table[:, h].clone().requires_grad_(step) if biased else None
            x = a @ b.T * s["scale"]
            if biased:
                x = x + (torch.take(t, bucket) if not step else _Lookup.apply(t, bucket))
            if causal:
                x = x.masked_fill(j > i, -math.inf)
            z = torch.logsumexp(x, 1)
            y = torch.exp(x - z[:, None]) @ c
            out[q0:q0 + n, h], lse[q0:q0 + n, h] = y.detach(), z.detach()
            if step:
                y.backward(s["dout"][q0:q0 + n, h].double())
                grads[0][q0:q0 + n, h] = a.grad
                grads[1][k0:k0 + m, h // groups] += b.grad
                grads[2][k0:k0 + m, h // groups] += c.grad
                if biased:
                    grads[3][:, h] += t.grad
        q0, k0 = q0 + n, k0 + m
    if not step:
        return {"out": out}
    return {"out": out, "lse": lse, **dict(zip(("dq", "dk", "dv", "d_rel_table"), grads))}


def _exact_append(s):
    """Token by token: token t of a request goes to row t % page of its page t / page."""
    table, pages = s["table"].tolist(), [s["k_pages"].double(), s["v_pages"].double()]
    to = [(table[b][t // s["page"]], t % s["page"])
          for b, (n, m) in enumerate(zip(s["lengths"], s["keys"])) for t in range(m - n, m)]
    page, row = (torch.tensor(x, device="cuda") for x in zip(*to))
    for into, new in zip(pages, (s["k"], s["v"])):
        into[page, row] = new.double()
    return {"k_pages": pages[0], "v_pages": pages[1]}


class _Lookup(torch.autograd.Function):
    """table[bucket], its gradient summed bucket by bucket (no scattered additions)."""

    @staticmethod
    def forward(ctx, table, bucket):
        ctx.save_for_backward(bucket)
        ctx.count = table.numel()
        return table[bucket]

    @staticmethod
    def backward(ctx, grad):
        bucket, = ctx.saved_tensors
        return torch.stack([torch.where(bucket == b, grad, 0.0).sum()
                            for b in range(ctx.count)]), None
