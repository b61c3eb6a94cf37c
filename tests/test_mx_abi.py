"""CPU-side refusals of the calls on an 8- or 4-bit cache: every documented status before anything
is launched (fake host addresses, no call here reaches the GPU), and the tensor-level checks."""
import ctypes

import pytest
import torch

import paper_2607_22696_amd as dsa
from paper_2607_22696_amd import _binding as B
from paper_2607_22696_amd import ops

CACHE = ["ck", "cv", "ck_scales", "cv_scales"]
FORWARD = ["q", *CACHE, "pages", "kv_lens", "cu_q", "bias_table", "bias_map", "out", "lse",
           "workspace"]
ROWS = ["k", "v", "cu_q", "kv_lens", "pages", *CACHE]


def addresses(names):
    return {n: (1 << 40) + i * (1 << 34) for i, n in enumerate(names)}


def desc(**kw):
    d = dict(batch=2, total_q=2, heads=4, kv_heads=2, head_dim=64, num_pages=100, page_size=16,
             max_pages=64, dtype="bf16", rel_min=-8, rel_span=9, rel_buckets=6)
    d.update(kw)
    return dsa.make_paged_desc(**d)


def cache_of(a, bits):
    return dsa.make_mx_cache(*[a[n] for n in CACHE], bits)


def forward(d=None, workspace_bytes=1 << 30, bits=8, cache=True, **over):
    a = addresses(FORWARD)
    a.update(over)
    return dsa.dsa3d_paged_forward_mx(d or desc(), a["q"], cache_of(a, bits) if cache else None,
                                      *[a[n] for n in FORWARD[5:]],
                                      workspace_bytes=workspace_bytes, stream=0, check=False)


def append(d=None, bits=8, cache=True, **over):
    a = addresses(ROWS)
    a.update(over)
    return dsa.dsa3d_paged_append_mx(d or desc(), *[a[n] for n in ROWS[:5]],
                                     cache_of(a, bits) if cache else None, stream=0, check=False)


def read(d=None, bits=8, cache=True, **over):
    a = addresses(ROWS)
    a.update(over)
    return dsa.dsa3d_paged_read_mx(d or desc(), cache_of(a, bits) if cache else None, a["pages"],
                                   a["kv_lens"], a["cu_q"], a["k"], a["v"], stream=0, check=False)


def test_struct_layout():
    assert ctypes.sizeof(B.dsa3d_mx_cache) == 4 * 8 + 8


@pytest.mark.parametrize("call,tensors", ((forward, ("q", "out")), (append, ("k", "v")),
                                          (read, ("k", "v"))))
def test_refusals(call, tensors):
    for name in tensors + ("pages", "kv_lens", "cu_q", *CACHE):
        assert call(**{name: None}) == B.DSA3D_ERR_NULL_POINTER, name
    assert call(cache=False) == B.DSA3D_ERR_NULL_POINTER
    for bits in (0, 3, 6, 16, -8):
        assert call(bits=bits) == B.DSA3D_ERR_UNSUPPORTED, bits
    for bad in (dict(batch=0), dict(total_q=-1), dict(kv_heads=0), dict(num_pages=-1),
                dict(page_size=0), dict(max_pages=-1), dict(max_kv=-1), dict(scale=-1.0),
                dict(num_pages=1 << 20, page_size=1 << 12)):
        assert call(desc(**bad)) == B.DSA3D_ERR_INVALID_SHAPE, bad
    assert call(desc(head_dim=32)) == B.DSA3D_ERR_UNSUPPORTED
    a = addresses(FORWARD if call is forward else ROWS)
    for name in tensors + tuple(CACHE):
        assert call(**{name: a[name] + 8}) == B.DSA3D_ERR_MISALIGNED, name
    for name in ("pages", "kv_lens", "cu_q"):
        assert call(**{name: a[name] + 1}) == B.DSA3D_ERR_MISALIGNED, name


def test_forward_refusals():
    a = addresses(FORWARD)
    for bad in (dict(heads=3), dict(q_stride=100), dict(rel_span=0), dict(max_pages=1 << 28)):
        assert forward(desc(**bad)) == B.DSA3D_ERR_INVALID_SHAPE, bad
    for bad in (dict(rel_span=2049), dict(rel_buckets=257),
                dict(heads=64, kv_heads=1, rel_span=97)):
        assert forward(desc(**bad)) == B.DSA3D_ERR_UNSUPPORTED, bad
    for bits in (8, 4):
        need = dsa.dsa3d_paged_forward_mx_workspace_size(desc(), bits)
        assert need > 0
        assert forward(workspace_bytes=need - 1, bits=bits) == B.DSA3D_ERR_WORKSPACE
        assert forward(workspace=None, bits=bits) == B.DSA3D_ERR_WORKSPACE
        assert forward(workspace=a["workspace"] + 16, bits=bits) == B.DSA3D_ERR_MISALIGNED
        assert dsa.dsa3d_paged_forward_mx_workspace_size(desc(max_kv=16), bits) == 0
    assert dsa.dsa3d_paged_forward_mx_workspace_size(desc(), 6) == 0
    for out in ("out", "lse", "workspace"):
        for other in ("q", *CACHE, "pages", "kv_lens", "cu_q", "bias_table"):
            assert forward(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)
    # the last bytes of the cache: 100 pages of 2 heads x 16 rows x 64 bytes, or 32
    for bits, size in ((8, 204800), (4, 102400)):
        assert forward(bits=bits, lse=a["ck"] + size - 4) == B.DSA3D_ERR_ALIAS
    assert forward(lse=a["cv_scales"] + 100 * 2 * 16 * 2 - 4) == B.DSA3D_ERR_ALIAS


@pytest.mark.parametrize("call", (append, read))
def test_row_refusals(call):
    a = addresses(ROWS)
    assert call(desc(k_stride=120)) == B.DSA3D_ERR_INVALID_SHAPE
    assert call(desc(v_stride=132)) == B.DSA3D_ERR_INVALID_SHAPE
    outs = CACHE if call is append else ["k", "v"]
    for out in outs:
        for other in ROWS:
            if other != out:
                assert call(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def raises(fn, *want, **kw):
    with pytest.raises(ValueError) as e:
        fn(**kw)
    for w in want:
        assert w in str(e.value), (w, str(e.value))


def small(bits=8, D=64):
    return dsa.paged_cache_mx(5, 16, 2, D, bits, device="cpu")


def test_new_caches():
    assert [tuple(t.shape) for t in small()] == [(5, 2, 16, 64)] * 2 + [(5, 2, 16, 2)] * 2
    assert [tuple(t.shape) for t in small(4, 128)] == [(5, 2, 16, 64)] * 2 + [(5, 2, 16, 4)] * 2
    raises(dsa.paged_cache_mx, "bits: 6", num_pages=1, page_size=1, kv_heads=1, head_dim=64, bits=6)
    raises(dsa.paged_cache_mx, "head_dim: 96", num_pages=1, page_size=1, kv_heads=1, head_dim=96)


@pytest.mark.parametrize("bits", (8, 4))
def test_tensor_checks(bits):
    c = dict(cache=small(bits), pages=ints(2, 3), kv_lens=ints(2), cu_q=ints(3))
    p = dict(c, q=bf(9, 4, 64))
    raises(ops.paged_forward_mx, "q: not a CUDA tensor", **p)
    k, v, ks, vs = c["cache"]
    for name, bad, say in (("cache", (k, v, ks), "cache: expected"),
                           ("cache", (k, v, ks, vs.flatten()), "cache: expected"),
                           ("cache", (k, v[:4], ks, vs), "cache v: shape"),
                           ("cache", (k, v, ks, vs.int()), "cache v_scales: dtype"),
                           ("cache", (k[..., :24], v, ks, vs), "cache k: shape"),
                           ("cache", (k, v, ks.transpose(1, 2), vs), "cache k_scales: shape"),
                           ("pages", ints(2), "pages: expected"), ("pages", ints(3, 3), "pages: shape"),
                           ("kv_lens", ints(3), "kv_lens: shape"), ("q", bf(9, 3, 64), "cache: 2 heads"),
                           ("q", bf(9, 4, 128), "cache: 2 heads"), ("cu_q", None, "cu_q: expected"),
                           ("max_kv", 2 ** 32, "does not fit"), ("workspace", bf(4), "workspace: dtype"),
                           ("out", bf(9, 4, 32), "out: shape"), ("q", bf(9, 4, 64).half(), "unsupported")):
        raises(ops.paged_forward_mx, say, **dict(p, **{name: bad}))
    r = dict(c, k=bf(9, 2, 64), v=bf(9, 2, 64))
    raises(ops.paged_append_mx, "k: not a CUDA tensor", **r)
    raises(ops.paged_append_mx, "v: expected", **dict(r, v=bf(8, 2, 64)))
    raises(ops.paged_append_mx, "k: expected", **dict(r, k=bf(9, 4, 64)))
    raises(ops.paged_append_mx, "k: unsupported dtype", **dict(r, k=bf(9, 2, 64).half()))
    raises(ops.paged_append_mx, "v: rows overlap", **dict(r, v=bf(1, 2, 64).expand(9, 2, 64)))
    raises(ops.paged_read_mx, "cu_q: not a CUDA tensor", rows=9, **c)
    raises(ops.paged_read_mx, "dtype: unsupported", rows=9, dtype=torch.float16, **c)
    raises(ops.paged_read_mx, "rows: -1", rows=-1, **c)
    raises(ops.paged_read_mx, "k: expected", rows=9, k=bf(8, 2, 64), **c)
    raises(ops.paged_read_mx, "v: expected", rows=9, v=torch.zeros(9, 2, 64), **c)
