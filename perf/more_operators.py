"""Performance cases of the quantised paged cache: its write, its reading back and its attention.

A cache of keys and values is read whole for every token that a language model writes, so its
bytes are the time.  Held in 8 or 4 bits it has half or a quarter of them: blocks of 32 channels
of one token and head share a power of two, the elements are e4m3 or e2m1 floats.  Three
operators, each in the form that a program which holds its tensors on the GPU runs:

  `store`  the newest tokens' keys and values quantised into the pages, and read back as they are
           held there, so that a prompt's own attention sees what later tokens will see
  `read`   tokens of the cache read back as packed rows
  `attend` attention of the newest tokens of each request over all that the pages hold

With `own` false every pass is computed in elementary torch operations in 32 bits, rounded once;
with `own` true it makes the library's calls.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ITEM = {"bf16": 2, "f32": 4}
_BLOCK = 32                          # channels that share a power of two
_LEAST = -117                        # the least power of two
_LARGEST = {8: 448.0, 4: 6.0}        # the largest element
_BUCKETS, _MAX_DISTANCE = 32, 128


# ----------------------------------------------------------------------------- cases

def _case(name, op, new, held, heads, kv_heads, head_dim, page, bits, dtype, bias=False):
    """`new`: tokens of each request in this call; `held`: all its tokens, those included."""
    return {"name": name, "op": op, "new": new, "held": held, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "bits": bits,
            "dtype": dtype, "bias": bias}


def _text(numbers):
    return " ".join(str(n) for n in numbers)


def _spread(count, lo, hi):
    """`count` lengths between lo and hi, uneven and in no order."""
    return [lo + (hi - lo) * ((7 * i + 3) % count) // max(count - 1, 1) for i in range(count)]


def listed():
    ones = _text([1] * 64)
    return [
        # the cache's side of a writing step of 64 users
        _case("store_decode_64", "store", ones, _text(_spread(64, 20, 500)), 32, 8, 128, 16, 8,
              "bf16"),
        # a small model in fp32, odd lengths, pages that no tile fits
        _case("store_f32_odd", "store", "700 1 33 259", "901 5 33 1259", 6, 2, 64, 24, 8, "f32"),
        # prompts read in, held in 4 bits
        _case("store_prompts_4bit", "store", "4096 1000 2500 1", "4096 1500 6000 900", 32, 8, 128,
              64, 4, "bf16"),
        # a few requests' caches as rows, to attend to them with other queries
        _case("read_prompts", "read", "2000 300 17 5000", "2000 450 17 7001", 16, 4, 128, 16, 8,
              "bf16"),
        # a long conversation taken up again, from 4 bits
        _case("read_long_4bit", "read", "60000", "60000", 32, 8, 128, 64, 4, "bf16"),
        # writing one token for one user: the shortest serving step
        _case("one_request", "attend", "1", "700", 32, 8, 128, 16, 8, "bf16"),
        # writing one token each for 64 users whose caches differ in length
        _case("decode_64", "attend", ones, _text(_spread(64, 200, 8000)), 32, 8, 128, 16, 8,
              "bf16"),
        # the same from 4 bits
        _case("decode_64_4bit", "attend", ones, _text(_spread(64, 200, 8000)), 32, 8, 128, 16, 4,
              "bf16"),
        # four users at the end of very long texts
        _case("long_4bit", "attend", "1 1 1 1", "120000 90001 31000 64000", 16, 2, 128, 64, 4,
              "bf16"),
        # drafts of a few tokens checked at once, 64 channels
        _case("drafts_64ch", "attend", _text([5] * 16), _text(_spread(16, 900, 6000)), 16, 4, 64,
              32, 8, "bf16"),
        # a small biased model in fp32, every head with its own keys
        _case("bias_f32_4bit", "attend", _text([1, 3] * 6), _text(_spread(12, 100, 4000)), 12, 12,
              64, 16, 4, "f32", True),
        # reading prompts in chunks beside users that are being written to, long caches
        _case("chunks", "attend", "512 1 801 1 1 300", "16000 3001 801 77 9000 5000", 32, 8, 128,
              64, 8, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((1, 1), (6, 6), (16, 16), (8, 2), (12, 4), (32, 8), (16, 2), (16, 1))


def draw(rng):
    op = rng.choice(("store", "read", "attend", "attend", "attend"))
    heads, kv_heads = rng.choice(_HEADS)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    head_dim, bits = rng.choice((64, 128)), rng.choice((8, 4))
    page = rng.choice((16, 16, 24, 32, 64, 100, 128))
    if op == "attend":
        count = _log_int(rng, 1, 64)
        chunk = rng.choice((1, 1, 6, 900))
        new = [_log_int(rng, 1, chunk) for _ in range(count)]
        longest = 8000 if chunk > 6 or count > 4 else 120000
        held = [n + _log_int(rng, 1, longest) for n in new]
        while sum(held) * kv_heads * head_dim > 250000 * 1024 or \
                len(new) * max(new) * max(held) * heads > 16384 ** 2 * 8:
            drop = held.index(max(held))
            del held[drop], new[drop]
            if not held:
                held, new = [300], [1]
    else:
        new = [_log_int(rng, 1, 6000) for _ in range(_log_int(rng, 1, 64))]
        while sum(new) * kv_heads * head_dim > 60000 * 1024:
            del new[new.index(max(new))]
        held = [n + rng.choice((0, _log_int(rng, 1, 1000))) for n in new]
    case = _case("", op, _text(new), _text(held), heads, kv_heads, head_dim, page, bits, dtype,
                 op == "attend" and rng.random() < 0.25)
    del case["name"]
    return case


# ----------------------------------------------------------------------------- 8 and 4 bits

def _two(power):
    """2^power as float32, exactly (a library's power function may be off by a rounding)."""
    return ((power + 127) << 23).to(torch.int32).view(torch.float32)


def _quantise(x, bits):
    """Codes and scale bytes of x [..., channels] in float32: a block's power of two is the least
    that puts its largest magnitude at the largest element or below."""
    blocks = x.unflatten(-1, (-1, _BLOCK))
    part, power = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    top_part, top_power = math.frexp(_LARGEST[bits])
    power = (power - top_power + (part > top_part)).clamp_min(_LEAST)
    y = blocks * _two(-power)
    size = y.abs()
    # the spacing of the elements around y: 3 bits behind the leading one from 2^-6 on, or 1 bit
    # from 1 on
    behind, least = (3, -6) if bits == 8 else (1, 0)
    lead = (torch.frexp(size)[1] - 1).clamp_min(least)
    size = torch.round(size * _two(behind - lead)).to(torch.int32)  # half to even
    # a whole number of spacings; 2 << behind of them are the next power of two's
    code = torch.where(size == 0, 0, ((lead - least) << behind) + size)
    code = (code + (torch.signbit(y).int() << (bits - 1))).flatten(-2).to(torch.uint8)
    if bits == 4:
        code = code[..., 0::2] + (code[..., 1::2] << 4)
    return code, (power + 127).squeeze(-1).to(torch.uint8)


def _values(code, scales, bits):
    """What codes and scale bytes stand for, in float32."""
    if bits == 4:
        code = torch.stack((code & 15, code >> 4), -1).flatten(-2)
    behind, least = (3, -6) if bits == 8 else (1, 0)
    size = (code & ((1 << (bits - 1)) - 1)).int()
    lead = (size >> behind).clamp_min(1) - 1
    size = size - (lead << behind)  # in spacings, the leading one included
    x = size * _two(lead + least - behind)
    x = torch.where(code >> (bits - 1) == 1, -x, x).unflatten(-1, (-1, _BLOCK))
    return (x * _two(scales.int() - 127)[..., None]).flatten(-2)


# ----------------------------------------------------------------------------- inputs

def _numbers(text):
    return [int(n) for n in text.split()]


def _starts(lengths):
    total = [0]
    for n in lengths:
        total.append(total[-1] + n)
    return total


def _bucket_map():
    """Buckets of the distances 128 .. 0 behind the query: half of them exact, the rest widening
    with the logarithm up to the last.  Whole-number arithmetic, so that a distance at a border
    falls to its side."""
    exact_to = _BUCKETS // 2
    wide = _BUCKETS - exact_to

    def bucket(n):
        if n < exact_to:
            return n
        t = 0
        while t + 1 < wide and (n ** wide) * exact_to ** (t + 1) >= \
                (_MAX_DISTANCE ** (t + 1)) * exact_to ** wide:
            t += 1
        return exact_to + t

    return [bucket(n) for n in range(_MAX_DISTANCE, -1, -1)]


def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _keys(gen, shape):
    """Keys: a few channels of every head are several times as large as the others."""
    x = _normal(gen, shape)
    return x.mul_(torch.where(torch.arange(shape[-1], device="cuda") % 23 == 5, 4.0, 0.9))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, D, bits, page = _TYPES[case["dtype"]], case["head_dim"], case["bits"], case["page"]
    H, G = case["heads"], case["kv_heads"]
    new, held = _numbers(case["new"]), _numbers(case["held"])
    counts = [-(-n // page) for n in held]
    total = sum(counts)
    # pages are handed out as requests grow, so that a request's pages lie scattered
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32).cpu()
    table = torch.full((len(held), max(counts)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    state = {"case": case, "scale": 1.0 / math.sqrt(D), "new": new, "held": held,
             "cu": _ints(_starts(new)), "kv_lens": _ints(held), "pages": table.cuda()}
    codes = [torch.zeros(total, G, page, D * bits // 8, dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    scales = [torch.zeros(total, G, page, D // _BLOCK, dtype=torch.uint8, device="cuda")
              for _ in range(2)]
    state["cache"] = (*codes, *scales)
    if case["op"] == "store":
        state["k"] = _keys(gen, (sum(new), G, D)).to(dt)
        state["v"] = _normal(gen, (sum(new), G, D)).to(dt)
        return state
    some = max(1, (1 << 24) // (G * page * D))  # pages at a time
    for i, make in enumerate((_keys, _normal)):
        for p in range(0, total, some):
            count = min(some, total - p)
            codes[i][p:p + count], scales[i][p:p + count] = \
                _quantise(make(gen, (count, G, page, D)), bits)
    if case["op"] == "attend":
        # queries a little longer than unit length give rows with some keys that stand out
        state["q"] = _normal(gen, (sum(new), H, D), 1.2).to(dt)
        if case["bias"]:
            state.update(rel_buckets=_ints(_bucket_map()), rel_min=-_MAX_DISTANCE,
                         rel_table=_normal(gen, (_BUCKETS, H)))
    return state


# ----------------------------------------------------------------------------- one pass

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _own_store(s):
    import paper_2607_22696_amd as dsa
    dsa.paged_append_mx(s["k"], s["v"], s["cache"], s["pages"], s["kv_lens"], s["cu"])
    return _own_read(s)


def _own_read(s):
    import paper_2607_22696_amd as dsa
    k, v = dsa.paged_read_mx(s["cache"], s["pages"], s["kv_lens"], s["cu"], sum(s["new"]),
                             dtype=_TYPES[s["case"]["dtype"]])
    return {"k": k, "v": v}


def _own_attend(s):
    import paper_2607_22696_amd as dsa
    how = {}
    if s["case"]["bias"]:
        how.update(rel_table=s["rel_table"], rel_buckets=s["rel_buckets"], rel_min=s["rel_min"])
    out, lse = dsa.paged_forward_mx(s["q"], s["cache"], s["pages"], s["kv_lens"], s["cu"],
                                    scale=s["scale"], max_kv=max(s["held"]), need_lse=True, **how)
    return {"out": out, "lse": lse}


_OWN = {"store": _own_store, "read": _own_read, "attend": _own_attend}


def _rows(starts, counts, width):
    """Rows of a packed tensor as [request, width], and which of them are a request's own."""
    at = torch.arange(width, device="cuda")
    there = at < counts[:, None]
    return torch.where(there, starts[:, None] + at, 0).long(), there


def _places(s):
    """Page and row of each packed token: the newest tokens stand last."""
    new = s["cu"].diff()
    rows, there = _rows(s["cu"][:-1], new, max(s["new"]))
    pos = torch.where(there, torch.arange(rows.shape[1], device="cuda") +
                      (s["kv_lens"] - new)[:, None], 0)
    page = s["pages"].gather(1, (pos // s["case"]["page"]).long()).long()
    return page[there], (pos % s["case"]["page"]).long()[there], rows[there]


def _plain_store(s):
    page, row, at = _places(s)
    for codes, scales, x in zip(s["cache"][:2], s["cache"][2:], (s["k"], s["v"])):
        c, e = _quantise(x[at].float(), s["case"]["bits"])
        codes.transpose(1, 2)[page, row] = c
        scales.transpose(1, 2)[page, row] = e
    return _plain_read(s)


def _plain_read(s):
    page, row, at = _places(s)
    got = []
    for codes, scales in zip(s["cache"][:2], s["cache"][2:]):
        x = _values(codes.transpose(1, 2)[page, row], scales.transpose(1, 2)[page, row],
                    s["case"]["bits"])
        got.append(torch.empty(x.shape, dtype=_TYPES[s["case"]["dtype"]], device="cuda"))
        got[-1][at] = x.to(got[-1].dtype)
    return {"k": got[0], "v": got[1]}


def _tokens(s, which):
    """All held keys (0) or values (1) as [request, kv_heads, tokens, head_dim] in 32 bits, zeros
    behind a request's last."""
    case, width = s["case"], max(s["held"])
    count = -(-width // case["page"])
    pages = s["pages"][:, :count].clamp_min(0).long()
    x = _values(s["cache"][which][pages], s["cache"][2 + which][pages], case["bits"])
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :width]
    there = torch.arange(width, device="cuda") < s["kv_lens"][:, None]
    return torch.where(there[:, None, :, None], x, 0.0)


def _plain_attend(s):
    case = s["case"]
    G, group = case["kv_heads"], case["heads"] // case["kv_heads"]
    new = s["cu"].diff()
    rows, there = _rows(s["cu"][:-1], new, max(s["new"]))
    B, n = rows.shape
    k, v = _tokens(s, 0), _tokens(s, 1)
    m = k.shape[2]
    q = s["q"][rows].float().transpose(1, 2).unflatten(1, (G, group)).flatten(2, 3).contiguous()
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    logits = logits.unflatten(2, (group, n))  # [request, key head, head of its group, query, key]
    pos = torch.arange(n, device="cuda") + (s["kv_lens"] - new)[:, None]
    ahead = torch.arange(m, device="cuda") - pos[:, :, None]
    if case["bias"]:
        at = s["rel_buckets"][(ahead - s["rel_min"]).clamp(0, s["rel_buckets"].numel() - 1)].long()
        logits += s["rel_table"][at].permute(0, 3, 1, 2).unflatten(1, (G, group))
    logits.masked_fill_((ahead > 0)[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = logits.sub_(top).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.div_(total).flatten(2, 3), v).unflatten(2, (group, n))
    lse = (top + torch.log(total))[..., 0]
    result = {"out": torch.empty_like(s["q"]),
              "lse": torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")}
    result["out"][rows[there]] = out.flatten(1, 2).transpose(1, 2)[there].to(s["q"].dtype)
    result["lse"][rows[there]] = lse.flatten(1, 2).transpose(1, 2)[there]
    return result


_PLAIN = {"store": _plain_store, "read": _plain_read, "attend": _plain_attend}


# ----------------------------------------------------------------------------- work

def work(case):
    item, H, G, D = _ITEM[case["dtype"]], case["heads"], case["kv_heads"], case["head_dim"]
    new, held = _numbers(case["new"]), _numbers(case["held"])
    token = 2 * G * (D * case["bits"] // 8 + D // _BLOCK)  # bytes of one token's keys and values
    rows = 2 * G * D * item
    if case["op"] == "store":  # rows in, tokens and rows out
        return {"bytes": sum(new) * (2 * rows + token), "flops": 0}
    if case["op"] == "read":
        return {"bytes": sum(new) * (rows + token), "flops": 0}
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(new, held))
    return {"bytes": sum(new) * H * (2 * D * item + 4) + sum(held) * token,
            "flops": 4 * pairs * H * D}


# ----------------------------------------------------------------------------- in 64 bits

def _elements(bits):
    """The elements that are not negative, in the order of their codes."""
    behind, bias, count = (3, 7, 127) if bits == 8 else (1, 1, 8)
    return torch.tensor([(c & ((1 << behind) - 1) if c >> behind == 0 else
                          (1 << behind) + (c & ((1 << behind) - 1))) *
                         2.0 ** (max(c >> behind, 1) - bias - behind) for c in range(count)],
                        dtype=torch.float64, device="cuda")


def _power(n):
    """2^n in float64, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _exact_rounded(x, bits):
    """x [rows, channels] in float64 as the cache holds it: the nearest element by search."""
    table = _elements(bits)
    x = x.unflatten(-1, (-1, _BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(top.clamp_min(2.0 ** -200) / table[-1]))
    power = torch.where(top > table[-1] * _power(power), power + 1, power)
    power = torch.where(top <= table[-1] * _power(power - 1), power - 1, power)
    scale = _power(power.clamp_min(_LEAST))
    y = x.abs() / scale
    above = torch.searchsorted(table, y.contiguous()).clamp_max(len(table) - 1)
    below = (above - 1).clamp_min(0)
    up, down = table[above] - y, y - table[below]
    pick = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    return (torch.sign(x) * table[pick] * scale).flatten(-2)


def _exact_held(s, b, which, first, last):
    """Tokens first .. last - 1 of request b from the codes, [tokens, kv_heads, head_dim]."""
    bits, page = s["case"]["bits"], s["case"]["page"]
    at = torch.arange(first, last, device="cuda")
    where = s["pages"][b].long()[at // page]
    code = s["cache"][which][where, :, at % page].long()
    if bits == 4:
        code = torch.stack((code % 16, code // 16), -1).flatten(-2)
    half = 1 << (bits - 1)
    x = _elements(bits)[code % half] * (1.0 - 2.0 * (code >= half))
    scale = _power(s["cache"][2 + which][where, :, at % page].long() - 127)
    return x * scale.repeat_interleave(_BLOCK, -1)


def exact(case, seed):
    """Request by request in float64."""
    s = prepare(case, seed)
    if case["op"] == "store":
        return {n: _exact_rounded(s[n].double(), case["bits"]) for n in ("k", "v")}
    if case["op"] == "read":
        return {n: torch.cat([_exact_held(s, b, i, m - t, m)
                              for b, (t, m) in enumerate(zip(s["new"], s["held"]))])
                for i, n in enumerate(("k", "v"))}
    group, bits_of = case["heads"] // case["kv_heads"], torch.float64
    out = torch.zeros(s["q"].shape, dtype=bits_of, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=bits_of, device="cuda")
    first = 0
    for b, (n, m) in enumerate(zip(s["new"], s["held"])):
        k, v = (_exact_held(s, b, i, 0, m) for i in (0, 1))
        i = torch.arange(n, device="cuda")[:, None] + (m - n)
        j = torch.arange(m, device="cuda")[None, :]
        for h in range(case["heads"]):
            x = (s["q"][first:first + n, h].double() @ k[:, h // group].T) * s["scale"]
            if case["bias"]:
                d = (j - i).clamp(-_MAX_DISTANCE, 0) + _MAX_DISTANCE
                x = x + s["rel_table"].double()[:, h][s["rel_buckets"].long()[d]]
            x = x.masked_fill(j > i, -math.inf)
            z = torch.logsumexp(x, 1)
            out[first:first + n, h] = torch.exp(x - z[:, None]) @ v[:, h // group]
            lse[first:first + n, h] = z
        first += n
    return {"out": out, "lse": lse}
