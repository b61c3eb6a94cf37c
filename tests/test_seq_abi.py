"""CPU-side refusals of the sequence calls: every documented status before anything is launched
(fake host addresses, no call here reaches the GPU), and the tensor-level checks."""
import ctypes

import pytest
import torch

import paper_2607_22696_amd as dsa
from paper_2607_22696_amd import _binding as B
from paper_2607_22696_amd import ops


def test_desc_layouts():
    assert ctypes.sizeof(B.dsa3d_seq_desc) == 12 * 4 + 3 * 8
    # 15 4-byte fields, padded to the strides' alignment
    assert ctypes.sizeof(B.dsa3d_paged_desc) == 16 * 4 + 3 * 8


def addresses(names):
    return {n: (1 << 40) + i * (1 << 34) for i, n in enumerate(names)}


SEQ = ["q", "k", "v", "cu_q", "cu_k", "bias_table", "bias_map", "out", "out_res", "lse"]
BACK = SEQ + ["dout", "dq", "dk", "dv", "d_table", "workspace"]


def seq_desc(**kw):
    d = dict(batch=2, total_q=100, total_k=100, heads=4, kv_heads=2, head_dim=64, dtype="bf16",
             rel_min=-8, rel_span=17, rel_buckets=6)
    d.update(kw)
    return dsa.make_seq_desc(**d)


def forward(desc=None, **over):
    a = addresses(SEQ)
    a.update(over)
    return dsa.dsa3d_seq_forward(desc or seq_desc(), *[a[n] for n in SEQ], stream=0, check=False)


def backward(desc=None, workspace_bytes=1 << 30, **over):
    a = addresses(BACK)
    a.update(over)
    order = [a[n] for n in SEQ] + [a[n] for n in ("dout", "dq", "dk", "dv", "d_table",
                                                  "workspace")]
    return dsa.dsa3d_seq_backward(desc or seq_desc(), *order, workspace_bytes=workspace_bytes,
                                  stream=0, check=False)


@pytest.mark.parametrize("call", (forward, backward))
def test_seq_refusals(call):
    for name in ("q", "k", "v", "cu_q", "out", "bias_table", "bias_map"):
        assert call(**{name: None}) == B.DSA3D_ERR_NULL_POINTER, name
    for bad in (dict(batch=0), dict(batch=1 << 24), dict(total_q=-1), dict(total_k=-1),
                dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan")), dict(head_dim=0),
                dict(total_q=1 << 30, total_k=1 << 30), dict(rel_span=0), dict(rel_buckets=-1),
                dict(rel_min=-(1 << 25)), dict(q_stride=255), dict(q_stride=257),
                dict(k_stride=127), dict(v_stride=129), dict(q_stride=-256)):
        assert call(seq_desc(**bad)) == B.DSA3D_ERR_INVALID_SHAPE, bad
    for bad in (dict(head_dim=32), dict(head_dim=256), dict(rel_span=2049),
                dict(rel_buckets=257)):
        assert call(seq_desc(**bad)) == B.DSA3D_ERR_UNSUPPORTED, bad
    d = seq_desc()
    d.dtype = 2
    assert call(d) == B.DSA3D_ERR_UNSUPPORTED
    d = seq_desc()
    d.causal = 2
    assert call(d) == B.DSA3D_ERR_INVALID_SHAPE
    # keys of their own without offsets; a residual for float32
    assert call(seq_desc(total_k=90), cu_k=None) == B.DSA3D_ERR_INVALID_SHAPE
    assert call(seq_desc(dtype="f32")) == B.DSA3D_ERR_UNSUPPORTED
    a = addresses(BACK)
    for name in ("q", "k", "v", "out", "out_res"):
        assert call(**{name: a[name] + 8}) == B.DSA3D_ERR_MISALIGNED, name
    for name in ("cu_q", "cu_k", "lse", "bias_table", "bias_map"):
        assert call(**{name: a[name] + 2}) == B.DSA3D_ERR_MISALIGNED, name


def test_seq_forward_aliases():
    a = addresses(SEQ)
    for out in ("out", "out_res", "lse"):
        for other in ("q", "k", "v", "cu_q", "cu_k", "bias_table", "bias_map"):
            assert forward(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)
    assert forward(out=a["lse"]) == B.DSA3D_ERR_ALIAS
    # the last row of a strided q: 99 strides and a row
    wide = seq_desc(q_stride=1024)
    assert forward(wide, out=a["q"] + (99 * 1024 + 256) * 2 - 16) == B.DSA3D_ERR_ALIAS


def test_seq_backward_refusals():
    a = addresses(BACK)
    for name in ("lse", "dout", "dq", "dk", "dv"):
        assert backward(**{name: None}) == B.DSA3D_ERR_NULL_POINTER, name
    for name in ("dout", "dq", "dk", "dv"):
        assert backward(**{name: a[name] + 4}) == B.DSA3D_ERR_MISALIGNED, name
    assert backward(d_table=a["d_table"] + 2) == B.DSA3D_ERR_MISALIGNED
    assert backward(workspace=a["workspace"] + 128) == B.DSA3D_ERR_MISALIGNED
    assert backward(workspace=None) == B.DSA3D_ERR_WORKSPACE
    need = dsa.dsa3d_seq_backward_workspace_size(seq_desc())
    assert need > 0 and backward(workspace_bytes=need - 1) == B.DSA3D_ERR_WORKSPACE
    assert backward(seq_desc(rel_buckets=0)) == B.DSA3D_ERR_INVALID_SHAPE  # no table to derive
    for out in ("dq", "dk", "dv", "d_table", "workspace"):
        for other in ("q", "v", "out", "out_res", "dout", "lse", "bias_table"):
            assert backward(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)
    assert backward(dq=a["dk"]) == B.DSA3D_ERR_ALIAS
    assert dsa.dsa3d_seq_backward_workspace_size(seq_desc(heads=0)) == 0


PAGED = ["q", "k_pages", "v_pages", "pages", "kv_lens", "cu_q", "bias_table", "bias_map", "out",
         "lse", "workspace"]
APPEND = ["k", "v", "cu_q", "kv_lens", "pages", "k_pages", "v_pages"]


def paged_desc(**kw):
    d = dict(batch=2, total_q=2, heads=4, kv_heads=2, head_dim=64, num_pages=100, page_size=16,
             max_pages=64, dtype="bf16", rel_min=-8, rel_span=9, rel_buckets=6)
    d.update(kw)
    return dsa.make_paged_desc(**d)


def paged(desc=None, workspace_bytes=1 << 30, **over):
    a = addresses(PAGED)
    a.update(over)
    return dsa.dsa3d_paged_forward(desc or paged_desc(), *[a[n] for n in PAGED],
                                   workspace_bytes=workspace_bytes, stream=0, check=False)


def append(desc=None, **over):
    a = addresses(APPEND)
    a.update(over)
    return dsa.dsa3d_paged_append(desc or paged_desc(), *[a[n] for n in APPEND], stream=0,
                                  check=False)


@pytest.mark.parametrize("call,tensors", ((paged, ("q", "k_pages", "v_pages")),
                                          (append, ("k", "v", "k_pages", "v_pages"))))
def test_paged_refusals(call, tensors):
    for name in tensors + ("pages", "kv_lens", "cu_q"):
        assert call(**{name: None}) == B.DSA3D_ERR_NULL_POINTER, name
    for bad in (dict(batch=0), dict(total_q=-1), dict(kv_heads=0), dict(num_pages=-1),
                dict(page_size=0), dict(max_pages=-1), dict(max_kv=-1), dict(scale=-1.0),
                dict(num_pages=1 << 20, page_size=1 << 12)):
        assert call(paged_desc(**bad)) == B.DSA3D_ERR_INVALID_SHAPE, bad
    assert call(paged_desc(head_dim=32)) == B.DSA3D_ERR_UNSUPPORTED
    a = addresses(PAGED if call is paged else APPEND)
    for name in tensors:
        assert call(**{name: a[name] + 8}) == B.DSA3D_ERR_MISALIGNED, name
    for name in ("pages", "kv_lens", "cu_q"):
        assert call(**{name: a[name] + 1}) == B.DSA3D_ERR_MISALIGNED, name


def test_paged_forward_refusals():
    a = addresses(PAGED)
    for bad in (dict(heads=3), dict(q_stride=100), dict(rel_span=0), dict(max_pages=1 << 28)):
        assert paged(paged_desc(**bad)) == B.DSA3D_ERR_INVALID_SHAPE, bad
    for bad in (dict(rel_span=2049), dict(rel_buckets=257),
                dict(heads=64, kv_heads=1, rel_span=97)):
        assert paged(paged_desc(**bad)) == B.DSA3D_ERR_UNSUPPORTED, bad
    need = dsa.dsa3d_paged_forward_workspace_size(paged_desc())
    assert need > 0
    assert paged(workspace_bytes=need - 1) == B.DSA3D_ERR_WORKSPACE
    assert paged(workspace=None) == B.DSA3D_ERR_WORKSPACE
    assert paged(workspace=a["workspace"] + 16) == B.DSA3D_ERR_MISALIGNED
    assert dsa.dsa3d_paged_forward_workspace_size(paged_desc(max_kv=16)) == 0
    for out in ("out", "lse", "workspace"):
        for other in ("q", "k_pages", "v_pages", "pages", "kv_lens", "cu_q", "bias_table"):
            assert paged(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)


def test_append_refusals():
    a = addresses(APPEND)
    assert append(paged_desc(k_stride=120)) == B.DSA3D_ERR_INVALID_SHAPE
    assert append(paged_desc(v_stride=132)) == B.DSA3D_ERR_INVALID_SHAPE
    for out in ("k_pages", "v_pages"):
        for other in ("k", "v", "cu_q", "kv_lens", "pages"):
            assert append(**{out: a[other]}) == B.DSA3D_ERR_ALIAS, (out, other)
    assert append(v_pages=a["k_pages"]) == B.DSA3D_ERR_ALIAS


def test_bucket_refusals():
    for bad in ((0, 128, 0), (1, 128, 0), (31, 128, 1), (2, 128, 1), (32, 8, 1), (32, 16, 0),
                (32, 0, 0), (32, -5, 0)):
        assert dsa.dsa3d_relative_buckets(*bad, check=False) == (None, B.DSA3D_ERR_INVALID_SHAPE)
    for bad in ((32, 1024, 1), (32, 2048, 0), (258, 600, 1)):
        assert dsa.dsa3d_relative_buckets(*bad, check=False) == (None, B.DSA3D_ERR_UNSUPPORTED)
    with pytest.raises(dsa.Dsa3dError):
        dsa.relative_buckets(1, 128, False, device="cpu")


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def raises(fn, *want, **kw):
    with pytest.raises(ValueError) as e:
        fn(**kw)
    for w in want:
        assert w in str(e.value), (w, str(e.value))


def test_tensor_checks():
    a = dict(q=bf(9, 4, 64), k=bf(9, 2, 64), v=bf(9, 2, 64), cu_q=ints(3))
    f32 = lambda *s: torch.zeros(s)  # noqa: E731
    raises(ops.seq_forward, "q: not a CUDA tensor", **a)
    for name, bad, say in (("q", f32(9, 4, 64).double(), "q: unsupported dtype"),
                           ("q", bf(9, 256), "q: expected [rows, heads, head_dim]"),
                           ("k", bf(9, 128), "k: expected a [rows"), ("k", bf(8, 2, 64), "no cu_k"),
                           ("k", bf(9, 3, 64), "do not divide"), ("k", f32(9, 2, 64), "k: expected"),
                           ("v", bf(8, 2, 64), "v: expected"), ("v", bf(9, 2, 32), "v: expected"),
                           ("k", bf(9, 64, 2).transpose(1, 2), "channels of a row"),
                           ("cu_q", ints(1), "cu_q: expected"),
                           ("cu_q", ints(3).long(), "cu_q: dtype"), ("cu_k", ints(4), "cu_k: shape"),
                           ("rel_table", f32(6, 3), "rel_table: shape"),
                           ("rel_buckets", ints(5), "without rel_table"),
                           ("lse", f32(9, 3), "lse: shape"), ("out", f32(9, 4, 64), "out: dtype")):
        kw = dict(a, **{name: bad})
        if name == "rel_table":
            kw["rel_buckets"] = ints(5)
        raises(ops.seq_forward, say, **kw)
    raises(ops.seq_forward, "out_res: dtype", out_res=f32(9, 4, 64), need_residual=True, **a)
    b = dict(a, out=bf(9, 4, 64), out_res=None, lse=f32(9, 4), dout=bf(9, 4, 64))
    raises(ops.seq_backward, "dout: shape", **dict(b, dout=bf(9, 2, 64)))
    raises(ops.seq_backward, "dout: not contiguous",
           **dict(b, dout=bf(9, 64, 4).transpose(1, 2)))
    raises(ops.seq_backward, "grads: expected (dq, dk, dv)", grads=(bf(1),) * 4, **b)
    raises(ops.seq_backward, "dk: shape", grads=(bf(9, 4, 64),) * 3, **b)
    raises(ops.seq_backward, "workspace: dtype", workspace=f32(4), **b)


def test_cache_checks():
    c = dict(k_pages=bf(5, 16, 2, 64), v_pages=bf(5, 16, 2, 64), pages=ints(2, 3), kv_lens=ints(2),
             cu_q=ints(3))
    p = dict(c, q=bf(9, 4, 64))
    raises(ops.paged_forward, "q: not a CUDA tensor", **p)
    for name, bad, say in (("k_pages", bf(5, 2, 64), "k_pages: expected"),
                           ("v_pages", bf(5, 16, 2, 32), "v_pages: shape"),
                           ("pages", ints(2), "pages: expected"), ("pages", ints(3, 3), "pages: shape"),
                           ("kv_lens", ints(3), "kv_lens: shape"), ("q", bf(9, 3, 64), "k_pages: 2 heads"),
                           ("q", bf(9, 4, 128), "k_pages: 2 heads"), ("cu_q", None, "cu_q: expected")):
        raises(ops.paged_forward, say, **dict(p, **{name: bad}))
    k = dict(c, k=bf(9, 2, 64), v=bf(9, 2, 64))
    raises(ops.paged_append, "k: not a CUDA tensor", **k)
    raises(ops.paged_append, "v: expected", **dict(k, v=bf(8, 2, 64)))
    raises(ops.paged_append, "k: expected", **dict(k, k=bf(9, 4, 64)))
    raises(ops.paged_append, "k: unsupported dtype", **dict(k, k=bf(9, 2, 64).half()))


def test_rows_that_overlap():
    """A row stride of 0 in a descriptor selects the row itself, so a broadcast tensor is refused
    before it gets there, as is every stride below a row."""
    wide = torch.zeros(4096, dtype=torch.bfloat16)
    a = dict(q=bf(9, 4, 64), k=bf(9, 2, 64), v=bf(9, 2, 64), cu_q=ints(3))
    for name, heads in (("q", 4), ("k", 2), ("v", 2)):
        for t in (bf(1, heads, 64).expand(9, heads, 64),
                  wide.as_strided((9, heads, 64), (64, 64, 1))):
            raises(ops.seq_forward, f"{name}: rows overlap", **dict(a, **{name: t}))
    c = dict(k_pages=bf(5, 16, 2, 64), v_pages=bf(5, 16, 2, 64), pages=ints(2, 3), kv_lens=ints(2),
             cu_q=ints(3))
    raises(ops.paged_forward, "q: rows overlap", q=bf(1, 4, 64).expand(9, 4, 64), **c)
    raises(ops.paged_append, "v: rows overlap", k=bf(9, 2, 64), v=bf(1, 2, 64).expand(9, 2, 64),
           **c)


def test_numbers_past_32_bits():
    c = dict(k_pages=bf(5, 16, 2, 64), v_pages=bf(5, 16, 2, 64), pages=ints(2, 3), kv_lens=ints(2),
             cu_q=ints(3), q=bf(9, 4, 64))
    raises(ops.paged_forward, "max_kv: 4294967296 does not fit", max_kv=2 ** 32, **c)
    a = dict(q=bf(9, 4, 64), k=bf(9, 2, 64), v=bf(9, 2, 64), cu_q=ints(3))
    raises(ops.seq_forward, "rel_min: -4294967296 does not fit", rel_min=-2 ** 32,
           rel_table=torch.zeros(6, 4), rel_buckets=ints(5), **a)
    raises(ops.relative_buckets, "max_distance: 4294967424", max_distance=2 ** 32 + 128)
