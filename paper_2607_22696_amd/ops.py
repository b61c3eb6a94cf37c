"""Tensor-level calls of the C ABI: check and allocate tensors with torch, then call the library.

q, k, v (and dout) are [B, T, H, W, heads, head_dim] CUDA tensors in float32 or bfloat16;
offsets are float32 [B, T, H, W, heads, P, 3] with (x, y, z) = (w, h, t) in token units.

The C ABI sees raw device pointers only and cannot know how large a buffer is, so every
tensor handed to it is checked here first (device, dtype, shape, contiguity): a wrong one
raises ValueError before anything is launched.
"""
from __future__ import annotations

import torch

from ._binding import (dsa3d_backward, dsa3d_backward_timed, dsa3d_backward_workspace_size,
                       dsa3d_dwconv3d_backward, dsa3d_dwconv3d_backward_workspace_size,
                       dsa3d_dwconv3d_forward, dsa3d_forward, dsa3d_paged_append,
                       dsa3d_paged_forward, dsa3d_paged_forward_workspace_size, dsa3d_pw_backward,
                       dsa3d_pw_backward_workspace_size, dsa3d_pw_forward, dsa3d_relative_buckets,
                       dsa3d_seq_backward, dsa3d_seq_backward_workspace_size, dsa3d_seq_forward,
                       dsa3d_win_backward, dsa3d_win_backward_workspace_size, dsa3d_win_forward,
                       make_conv_desc, make_desc, make_paged_desc, make_seq_desc, make_win_desc)

_IO_DTYPES = {torch.bfloat16: "bf16", torch.float32: "f32"}


class _Checks:
    """Collects every problem with the arguments of one call, then raises them together."""

    def __init__(self, where):
        self.where = where
        self.problems = []

    def tensor(self, name, t, shape, dtype, device):
        if isinstance(t, torch.Tensor) and t.dtype == dtype and t.shape == shape and \
                t.device == device and t.is_contiguous():
            return
        if not isinstance(t, torch.Tensor):
            self.problems.append(f"{name}: expected a tensor, got {type(t).__name__}")
            return
        bad = []
        if t.dtype != dtype:
            bad.append(f"dtype {t.dtype} (expected {dtype})")
        if tuple(t.shape) != tuple(shape):
            bad.append(f"shape {tuple(t.shape)} (expected {tuple(shape)})")
        if not t.is_contiguous():
            bad.append("not contiguous")
        if t.device != device:
            bad.append(f"on {t.device} (expected {device})")
        if bad:
            self.problems.append(f"{name}: " + ", ".join(bad))

    def workspace(self, t, device):
        if t is not None:
            n = t.numel() if isinstance(t, torch.Tensor) else 0
            self.tensor("workspace", t, (n,), torch.uint8, device)

    def optional(self, name, t, shape, dtype, device):
        if t is not None:
            self.tensor(name, t, shape, dtype, device)

    def done(self):
        if self.problems:
            raise ValueError(f"{self.where}: " + "; ".join(self.problems))


def _lead(chk, name, x, ndim, what, dtypes=_IO_DTYPES):
    """The tensor that fixes shape, dtype and device of a call: a CUDA tensor of `ndim` dims in
    one of `dtypes`.  Returns its device; raises at once when the other tensors cannot be
    checked against it (not a tensor, wrong rank, unsupported dtype), else the remaining
    problems are collected with those of the other tensors."""
    if not isinstance(x, torch.Tensor):
        chk.problems.append(f"{name}: expected a tensor, got {type(x).__name__}")
        chk.done()
    if x.dim() != ndim:
        chk.problems.append(f"{name}: expected {what}, got shape {tuple(x.shape)}")
    if x.dtype not in dtypes:
        chk.problems.append(f"{name}: unsupported dtype {x.dtype}")
    chk.done()
    if not x.is_cuda:
        chk.problems.append(f"{name}: not a CUDA tensor ({x.device})")
    if not x.is_contiguous():
        chk.problems.append(f"{name}: not contiguous")
    return x.device


def _kernel(chk, kernel):
    try:
        kt, kh, kw = (int(a) for a in kernel)
    except (TypeError, ValueError):
        chk.problems.append(f"kernel: expected three odd sizes, got {kernel!r}")
        return 1, 1, 1
    return kt, kh, kw


def _desc(q, kernel, scale):
    B, T, H, W, heads, D = q.shape
    kt, kh, kw = kernel
    return make_desc(B, T, H, W, heads, D, kt, kh, kw, _IO_DTYPES[q.dtype], scale)


def forward(q, k, v, offsets, kernel=(3, 3, 3), scale=0.0, need_lse=True, out=None, lse=None):
    """Returns (out, lse); lse is None when need_lse is False."""
    chk = _Checks("forward")
    dev = _lead(chk, "q", q, 6, "[B, T, H, W, heads, head_dim]")
    kern = _kernel(chk, kernel)
    P = kern[0] * kern[1] * kern[2]
    for name, t in (("k", k), ("v", v)):
        chk.tensor(name, t, q.shape, q.dtype, dev)
    chk.tensor("offsets", offsets, tuple(q.shape[:5]) + (P, 3), torch.float32, dev)
    chk.optional("out", out, q.shape, q.dtype, dev)
    if need_lse:
        chk.optional("lse", lse, q.shape[:5], torch.float32, dev)
    chk.done()
    desc = _desc(q, kern, scale)
    if out is None:
        out = torch.empty_like(q)
    if need_lse and lse is None:
        lse = torch.empty(q.shape[:5], dtype=torch.float32, device=dev)
    dsa3d_forward(desc, q, k, v, offsets, out, lse if need_lse else None)
    return out, (lse if need_lse else None)


def backward(q, k, v, offsets, lse, dout, kernel=(3, 3, 3), scale=0.0, grads=None, workspace=None,
             phase_events=None, out=None):
    """Returns (dq, dk, dv, d_offsets), all float32.  `out` (the forward's output) is optional:
    the library forms Delta exactly without it.  `grads` = (dq, dk, dv, d_offsets) to write
    into.  `workspace` (a uint8 CUDA tensor) is allocated here when missing or too small.
    `phase_events`: optional list of DSA3D_BACKWARD_PHASES + 1 created torch.cuda.Event objects
    marking the phases (see dsa3d_backward_timed)."""
    chk = _Checks("backward")
    dev = _lead(chk, "q", q, 6, "[B, T, H, W, heads, head_dim]")
    kern = _kernel(chk, kernel)
    P = kern[0] * kern[1] * kern[2]
    off_shape = tuple(q.shape[:5]) + (P, 3)
    for name, t in (("k", k), ("v", v), ("dout", dout)):
        chk.tensor(name, t, q.shape, q.dtype, dev)
    chk.optional("out", out, q.shape, q.dtype, dev)
    chk.tensor("offsets", offsets, off_shape, torch.float32, dev)
    chk.tensor("lse", lse, q.shape[:5], torch.float32, dev)
    if grads is not None:
        if len(grads) != 4:
            chk.problems.append("grads: expected (dq, dk, dv, d_offsets)")
        else:
            for name, t in zip(("dq", "dk", "dv"), grads[:3]):
                chk.tensor(name, t, q.shape, torch.float32, dev)
            chk.tensor("d_offsets", grads[3], off_shape, torch.float32, dev)
    chk.workspace(workspace, dev)
    chk.done()
    desc = _desc(q, kern, scale)
    if grads is None:
        f32 = dict(dtype=torch.float32, device=dev)
        grads = (torch.empty(q.shape, **f32), torch.empty(q.shape, **f32),
                 torch.empty(q.shape, **f32), torch.empty(off_shape, **f32))
    dq, dk, dv, doff = grads
    need = dsa3d_backward_workspace_size(desc)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    if phase_events is None:
        dsa3d_backward(desc, q, k, v, offsets, out, lse, dout, dq, dk, dv, doff, workspace, need)
    else:
        dsa3d_backward_timed(desc, q, k, v, offsets, out, lse, dout, dq, dk, dv, doff, workspace,
                             need, events=phase_events)
    return dq, dk, dv, doff


def _conv_desc(chk, x, weight):
    dev = _lead(chk, "x", x, 5, "[B, T, H, W, C]")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 4:
        chk.problems.append("weight: expected a float32 [C, kt, kh, kw] tensor")
        chk.done()
    B, T, H, W, C = x.shape
    kt, kh, kw = weight.shape[1:]
    chk.tensor("weight", weight, (C, kt, kh, kw), torch.float32, dev)
    return dev, make_conv_desc(B, T, H, W, C, kt, kh, kw, _IO_DTYPES[x.dtype])


def dwconv3d_forward(x, weight, bias=None, out=None, accumulate=False):
    """Depthwise 3D convolution (the DWConv3D term of Eq. (1)): x [B,T,H,W,C] (bf16 or fp32),
    weight float32 [C,kt,kh,kw], bias float32 [C] or None.  Returns out (x's dtype); with
    accumulate=True the result is added to `out`."""
    chk = _Checks("dwconv3d_forward")
    dev, desc = _conv_desc(chk, x, weight)
    chk.optional("bias", bias, (x.shape[4],), torch.float32, dev)
    chk.optional("out", out, x.shape, x.dtype, dev)
    if accumulate and out is None:
        chk.problems.append("accumulate needs an output to add to")
    chk.done()
    if out is None:
        out = torch.empty_like(x)
    dsa3d_dwconv3d_forward(desc, x, weight, bias, out, accumulate)
    return out


def dwconv3d_backward(x, weight, dy, need_dx=True, need_dweight=True, need_dbias=True,
                      dx=None, accumulate_dx=False, workspace=None):
    """Returns (dx, dweight, dbias) as float32 (None where not requested)."""
    chk = _Checks("dwconv3d_backward")
    dev, desc = _conv_desc(chk, x, weight)
    chk.tensor("dy", dy, x.shape, x.dtype, dev)
    if need_dx:
        chk.optional("dx", dx, x.shape, torch.float32, dev)
        if accumulate_dx and dx is None:
            chk.problems.append("accumulate_dx needs a dx to add to")
    chk.workspace(workspace, dev)
    chk.done()
    f32 = dict(dtype=torch.float32, device=dev)
    if need_dx and dx is None:
        dx = torch.empty(x.shape, **f32)
    dx = dx if need_dx else None
    dw = torch.empty(weight.shape, **f32) if need_dweight else None
    db = torch.empty(weight.shape[0], **f32) if need_dbias else None
    need = 0
    if dw is not None or db is not None:
        need = dsa3d_dwconv3d_backward_workspace_size(desc)
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    dsa3d_dwconv3d_backward(desc, x, weight, dy, dx, dw, db, workspace, need, accumulate_dx)
    return dx, dw, db


def pw_forward(logits, v, offsets, kernel=(3, 3, 3), need_lse=True, out=None, lse=None):
    """Predicted-weights variant: softmax over the given logits [B,T,H,W,heads,P] (fp32)
    instead of q.k.  Returns (out, lse)."""
    chk = _Checks("pw_forward")
    dev = _lead(chk, "v", v, 6, "[B, T, H, W, heads, head_dim]")
    kern = _kernel(chk, kernel)
    P = kern[0] * kern[1] * kern[2]
    chk.tensor("logits", logits, tuple(v.shape[:5]) + (P,), torch.float32, dev)
    chk.tensor("offsets", offsets, tuple(v.shape[:5]) + (P, 3), torch.float32, dev)
    chk.optional("out", out, v.shape, v.dtype, dev)
    if need_lse:
        chk.optional("lse", lse, v.shape[:5], torch.float32, dev)
    chk.done()
    desc = _desc(v, kern, 0.0)
    if out is None:
        out = torch.empty_like(v)
    if need_lse and lse is None:
        lse = torch.empty(v.shape[:-1], dtype=torch.float32, device=dev)
    dsa3d_pw_forward(desc, logits, v, offsets, out, lse if need_lse else None)
    return out, (lse if need_lse else None)


def pw_backward(logits, v, offsets, lse, dout, kernel=(3, 3, 3), grads=None, workspace=None,
                phase_events=None):
    """Returns (dlogits, dv, d_offsets), float32.  `phase_events` as for backward()."""
    chk = _Checks("pw_backward")
    dev = _lead(chk, "v", v, 6, "[B, T, H, W, heads, head_dim]")
    kern = _kernel(chk, kernel)
    P = kern[0] * kern[1] * kern[2]
    lshape, oshape = tuple(v.shape[:5]) + (P,), tuple(v.shape[:5]) + (P, 3)
    chk.tensor("logits", logits, lshape, torch.float32, dev)
    chk.tensor("offsets", offsets, oshape, torch.float32, dev)
    chk.tensor("lse", lse, v.shape[:5], torch.float32, dev)
    chk.tensor("dout", dout, v.shape, v.dtype, dev)
    if grads is not None:
        if len(grads) != 3:
            chk.problems.append("grads: expected (dlogits, dv, d_offsets)")
        else:
            chk.tensor("dlogits", grads[0], lshape, torch.float32, dev)
            chk.tensor("dv", grads[1], v.shape, torch.float32, dev)
            chk.tensor("d_offsets", grads[2], oshape, torch.float32, dev)
    chk.workspace(workspace, dev)
    chk.done()
    desc = _desc(v, kern, 0.0)
    if grads is None:
        f32 = dict(dtype=torch.float32, device=dev)
        grads = (torch.empty(lshape, **f32), torch.empty(v.shape, **f32),
                 torch.empty(oshape, **f32))
    dlog, dv, doff = grads
    need = dsa3d_pw_backward_workspace_size(desc)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    dsa3d_pw_backward(desc, logits, v, offsets, lse, dout, dlog, dv, doff, workspace, need,
                      events=phase_events)
    return dlog, dv, doff


def _win_lead(chk, q):
    return _lead(chk, "q", q, 6, "[B, T, H, W, heads, head_dim]", {torch.bfloat16: "bf16"})


def win_forward(q, k, v, window=(3, 16, 16), shift=(0, 0, 0), scale=0.0, need_lse=True,
                need_residual=True, out=None, lse=None, out_res=None):
    """Fixed / shifted window attention (bf16).  Returns (out, lse, out_res); out_res, the bf16
    rounding residual of out that the backward uses for an exact Delta, is None when
    need_residual is False (and lse when need_lse is False)."""
    chk = _Checks("win_forward")
    dev = _win_lead(chk, q)
    for name, t in (("k", k), ("v", v)):
        chk.tensor(name, t, q.shape, q.dtype, dev)
    chk.optional("out", out, q.shape, q.dtype, dev)
    if need_lse:
        chk.optional("lse", lse, q.shape[:5], torch.float32, dev)
    if need_residual:
        chk.optional("out_res", out_res, q.shape, q.dtype, dev)
    chk.done()
    B, T, H, W, heads, D = q.shape
    desc = make_win_desc(B, T, H, W, heads, D, window, shift, "bf16", scale)
    if out is None:
        out = torch.empty_like(q)
    if need_lse and lse is None:
        lse = torch.empty(q.shape[:5], dtype=torch.float32, device=dev)
    if need_residual and out_res is None:
        out_res = torch.empty_like(q)
    dsa3d_win_forward(desc, q, k, v, out, out_res if need_residual else None,
                      lse if need_lse else None)
    return out, (lse if need_lse else None), (out_res if need_residual else None)


def win_backward(q, k, v, out, out_res, lse, dout, window=(3, 16, 16), shift=(0, 0, 0),
                 scale=0.0, grads=None, workspace=None, phase_events=None):
    """Returns (dq, dk, dv), float32.  out_res may be None (Delta from the rounded out alone).
    `phase_events`: optional DSA3D_WIN_BACKWARD_PHASES + 1 created torch.cuda.Event objects
    marking the two passes."""
    chk = _Checks("win_backward")
    dev = _win_lead(chk, q)
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout)):
        chk.tensor(name, t, q.shape, q.dtype, dev)
    chk.optional("out_res", out_res, q.shape, q.dtype, dev)
    chk.tensor("lse", lse, q.shape[:5], torch.float32, dev)
    if grads is not None:
        if len(grads) != 3:
            chk.problems.append("grads: expected (dq, dk, dv)")
        else:
            for name, t in zip(("dq", "dk", "dv"), grads):
                chk.tensor(name, t, q.shape, torch.float32, dev)
    chk.workspace(workspace, dev)
    chk.done()
    B, T, H, W, heads, D = q.shape
    desc = make_win_desc(B, T, H, W, heads, D, window, shift, "bf16", scale)
    if grads is None:
        f32 = dict(dtype=torch.float32, device=dev)
        grads = tuple(torch.empty(q.shape, **f32) for _ in range(3))
    dq, dk, dv = grads
    need = dsa3d_win_backward_workspace_size(desc)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    dsa3d_win_backward(desc, q, k, v, out, out_res, lse, dout, dq, dk, dv, workspace, need,
                       events=phase_events)
    return dq, dk, dv


# ----------------------------------------------------------------------------- packed sequences

def _rows(chk, name, t, heads, head_dim, dtype, device, rows=None):
    """Checks a packed [rows, heads, head_dim] tensor whose rows may lie any distance apart (a
    slice of a fused projection) and returns that distance in elements, 0 for none between."""
    if not isinstance(t, torch.Tensor):
        chk.problems.append(f"{name}: expected a tensor, got {type(t).__name__}")
        return 0
    shape = t.shape
    if shape == (rows, heads, head_dim) and t.dtype == dtype and t.device == device and \
            t.is_contiguous():
        return 0
    if t.dim() != 3 or shape[1] != heads or shape[2] != head_dim or \
            (rows is not None and shape[0] != rows) or t.dtype != dtype or t.device != device:
        want = ("rows" if rows is None else rows, heads, head_dim)
        chk.problems.append(f"{name}: expected {dtype} [{want[0]}, {want[1]}, {want[2]}] on "
                            f"{device}, got {t.dtype} {tuple(shape)} on {t.device}")
        return 0
    if t.is_contiguous():
        return 0
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != head_dim):
        chk.problems.append(f"{name}: heads and channels of a row must be contiguous")
        return 0
    if t.stride(0) < heads * head_dim:  # 0 would select a row's length
        chk.problems.append(f"{name}: rows overlap (stride {t.stride(0)})")
        return 0
    return t.stride(0)


def _ints(chk, name, t, shape, device):
    chk.tensor(name, t, shape, torch.int32, device)


def _int32(chk, name, x):
    """An int of the descriptor (ctypes would drop the bits above)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        chk.problems.append(f"{name}: {x} does not fit 32 bits")
    return x


def _cu(chk, name, t, device):
    """Checks a cu_seqlens tensor and returns the number of sequences."""
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.numel() < 2:
        chk.problems.append(f"{name}: expected an int32 tensor of sequences + 1 row offsets")
        chk.done()
    chk.tensor(name, t, t.shape, torch.int32, device)
    return t.numel() - 1


def _relative(chk, rel_table, rel_buckets, rel_min, heads, device):
    """Checks the bias arguments; returns (rel_min, rel_span, rel_buckets) of the descriptor."""
    if rel_table is None:
        if rel_buckets is not None:
            chk.problems.append("rel_buckets: given without rel_table")
        return 0, 0, 0
    if not isinstance(rel_table, torch.Tensor) or rel_table.dim() != 2:
        chk.problems.append("rel_table: expected a float32 [buckets, heads] tensor")
        chk.done()
    chk.tensor("rel_table", rel_table, (rel_table.shape[0], heads), torch.float32, device)
    if not isinstance(rel_buckets, torch.Tensor) or rel_buckets.dim() != 1:
        chk.problems.append("rel_buckets: expected an int32 tensor, one bucket per distance")
        chk.done()
    _ints(chk, "rel_buckets", rel_buckets, tuple(rel_buckets.shape), device)
    if rel_table.shape[0] < 1 or rel_buckets.numel() < 1:
        chk.problems.append("rel_table, rel_buckets: empty")
    return _int32(chk, "rel_min", rel_min), rel_buckets.numel(), rel_table.shape[0]


def _lead_rows(chk, q):
    """The tensor that fixes type, heads and device of a call on packed rows."""
    if not isinstance(q, torch.Tensor):
        chk.problems.append(f"q: expected a tensor, got {type(q).__name__}")
        chk.done()
    if q.dim() != 3:
        chk.problems.append(f"q: expected [rows, heads, head_dim], got shape {tuple(q.shape)}")
    if q.dtype not in _IO_DTYPES:
        chk.problems.append(f"q: unsupported dtype {q.dtype}")
    chk.done()
    if not q.is_cuda:
        chk.problems.append(f"q: not a CUDA tensor ({q.device})")
    return q.device


# The current stream's handle, without the Stream object around it where torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(device, call, *args, **kw):
    """The call on the current stream of the tensors' device, with that device current."""
    index = device.index
    if index == torch.cuda.current_device():
        call(*args, stream=_raw_stream(index), **kw)
    else:
        with torch.cuda.device(device):
            call(*args, stream=_raw_stream(index), **kw)


def _like(t, device):
    """A new contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else \
        torch.empty(t.shape, dtype=t.dtype, device=device)


def relative_buckets(num_buckets=32, max_distance=128, both=True, device="cuda"):
    """The usual map of distances (key minus query position) to buckets: half of a direction's
    buckets hold one distance each, the others widen with the logarithm up to max_distance, from
    where on all distances share the last one.  With `both` keys ahead of the query have buckets
    of their own.  Returns (rel_buckets, rel_min) as the calls below take them."""
    chk = _Checks("relative_buckets")
    num_buckets = _int32(chk, "num_buckets", num_buckets)
    max_distance = _int32(chk, "max_distance", max_distance)
    chk.done()
    values, rel_min = dsa3d_relative_buckets(num_buckets, max_distance, both)
    return torch.tensor(values, dtype=torch.int32, device=device), rel_min


def _seq_desc(chk, q, k, v, cu_q, cu_k, causal, scale, rel_table, rel_buckets, rel_min):
    dev = _lead_rows(chk, q)
    nq, heads, D = q.shape
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        chk.problems.append("k: expected a [rows, heads, head_dim] tensor")
        chk.done()
    nk, kv_heads = k.shape[0], k.shape[1]
    if kv_heads < 1 or heads % kv_heads:
        chk.problems.append(f"k: {kv_heads} heads do not divide the {heads} of q")
    dtype = q.dtype
    qs = _rows(chk, "q", q, heads, D, dtype, dev, nq)
    ks = _rows(chk, "k", k, kv_heads, D, dtype, dev, nk)
    vs = _rows(chk, "v", v, kv_heads, D, dtype, dev, nk)
    batch = _cu(chk, "cu_q", cu_q, dev)
    if cu_k is not None:
        _ints(chk, "cu_k", cu_k, (batch + 1,), dev)
    elif nk != nq:
        chk.problems.append(f"k: {nk} rows, but q has {nq} and there is no cu_k")
    lo, span, buckets = _relative(chk, rel_table, rel_buckets, rel_min, heads, dev)
    return dev, make_seq_desc(batch, nq, nk, heads, kv_heads, D, causal, _IO_DTYPES[dtype],
                              scale, lo, span, buckets, qs, ks, vs)


def seq_forward(q, k, v, cu_q, cu_k=None, causal=False, scale=0.0, rel_table=None,
                rel_buckets=None, rel_min=0, need_lse=True, need_residual=False, out=None,
                lse=None, out_res=None):
    """Attention of packed sequences (bf16 or float32): q [rows, heads, head_dim], k and v
    [rows, kv_heads, head_dim], rows of a tensor any distance apart, sequence b in rows cu_q[b]
    .. cu_q[b + 1] - 1 (int32, on the GPU), its keys in those of cu_k (the same where None).
    `rel_table` (float32 [buckets, heads]) adds rel_table[rel_buckets[distance - rel_min]] to the
    logits, distances clamped to the ends of rel_buckets (see relative_buckets).
    Returns (out, lse, out_res).  out_res, the bf16 rounding residual of out, is what a bias
    gradient to some 2^-17 needs; it is None unless need_residual is set, and for float32
    tensors, which have none (as lse is None when need_lse is False)."""
    chk = _Checks("seq_forward")
    dev, desc = _seq_desc(chk, q, k, v, cu_q, cu_k, causal, scale, rel_table, rel_buckets, rel_min)
    need_residual = need_residual and q.dtype == torch.bfloat16
    chk.optional("out", out, q.shape, q.dtype, dev)
    if need_lse:
        chk.optional("lse", lse, q.shape[:2], torch.float32, dev)
    if need_residual:
        chk.optional("out_res", out_res, q.shape, q.dtype, dev)
    chk.done()
    if out is None:
        out = _like(q, dev)
    if not need_lse:
        lse = None
    elif lse is None:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=dev)
    if not need_residual:
        out_res = None
    elif out_res is None:
        out_res = _like(q, dev)
    _launch(dev, dsa3d_seq_forward, desc, q, k, v, cu_q, cu_k, rel_table, rel_buckets, out,
            out_res, lse)
    return out, lse, out_res


def seq_backward(q, k, v, out, out_res, lse, dout, cu_q, cu_k=None, causal=False, scale=0.0,
                 rel_table=None, rel_buckets=None, rel_min=0, need_table=True, grads=None,
                 workspace=None):
    """Returns (dq, dk, dv) in the type of q, and with rel_table also its gradient (float32; None
    where need_table is False).  `grads`: tensors to write into, in this order.  out_res may be
    None (Delta from the rounded out alone).  out, out_res and lse may be those of more keys than
    the call has (the keys of a sequence in several calls, joined): the gradients are sums over the
    call's keys."""
    chk = _Checks("seq_backward")
    dev, desc = _seq_desc(chk, q, k, v, cu_q, cu_k, causal, scale, rel_table, rel_buckets, rel_min)
    for name, t in (("out", out), ("dout", dout)):
        chk.tensor(name, t, q.shape, q.dtype, dev)
    chk.optional("out_res", out_res, q.shape, q.dtype, dev)
    chk.tensor("lse", lse, q.shape[:2], torch.float32, dev)
    count = 3 if rel_table is None else 4
    need_table = need_table and rel_table is not None
    if grads is not None:
        if len(grads) != count:
            chk.problems.append("grads: expected (dq, dk, dv" +
                                (", d_rel_table)" if count == 4 else ")"))
        else:
            for name, t, like in zip(("dq", "dk", "dv"), grads, (q, k, k)):
                chk.tensor(name, t, like.shape, q.dtype, dev)
            if need_table:
                chk.tensor("d_rel_table", grads[3], rel_table.shape, torch.float32, dev)
    chk.workspace(workspace, dev)
    chk.done()
    if grads is None:
        grads = [_like(x, dev) for x in (q, k, k)]
        if count == 4:
            grads.append(_like(rel_table, dev) if need_table else None)
    need = dsa3d_seq_backward_workspace_size(desc)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    d_table = grads[3] if need_table else None
    _launch(dev, dsa3d_seq_backward, desc, q, k, v, cu_q, cu_k, rel_table, rel_buckets, out,
            out_res, lse, dout, grads[0], grads[1], grads[2], d_table, workspace, need)
    return tuple(grads[:3]) if count == 3 else (*grads[:3], d_table)


# ----------------------------------------------------------------------------- a paged cache

def _pages(chk, k_pages, v_pages, pages, kv_lens, cu_q, dtype, device):
    """Checks the cache; returns (requests, num_pages, page_size, kv_heads, head_dim, columns)."""
    if not isinstance(k_pages, torch.Tensor) or k_pages.dim() != 4:
        chk.problems.append("k_pages: expected [pages, page_size, kv_heads, head_dim]")
        chk.done()
    shape = k_pages.shape
    chk.tensor("k_pages", k_pages, shape, dtype, device)
    chk.tensor("v_pages", v_pages, shape, dtype, device)
    batch = _cu(chk, "cu_q", cu_q, device)
    _ints(chk, "kv_lens", kv_lens, (batch,), device)
    if not isinstance(pages, torch.Tensor) or pages.dim() != 2:
        chk.problems.append("pages: expected an int32 [requests, columns] tensor")
        chk.done()
    _ints(chk, "pages", pages, (batch, pages.shape[1]), device)
    return (batch, *shape, pages.shape[1])


def paged_append(k, v, k_pages, v_pages, pages, kv_lens, cu_q):
    """Writes the new tokens' k, v [rows, kv_heads, head_dim] (packed by cu_q, rows any distance
    apart) into the pages k_pages, v_pages [pages, page_size, kv_heads, head_dim], in place.
    Request b holds kv_lens[b] tokens with the new ones, token j of them in row j % page_size of
    page pages[b, j // page_size]; a token whose page number is outside the tensors is dropped."""
    chk = _Checks("paged_append")
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        chk.problems.append("k: expected a [rows, kv_heads, head_dim] tensor")
        chk.done()
    if k.dtype not in _IO_DTYPES:
        chk.problems.append(f"k: unsupported dtype {k.dtype}")
        chk.done()
    if not k.is_cuda:
        chk.problems.append(f"k: not a CUDA tensor ({k.device})")
    dev = k.device
    batch, num, size, heads, D, columns = _pages(chk, k_pages, v_pages, pages, kv_lens, cu_q,
                                                 k.dtype, dev)
    ks = _rows(chk, "k", k, heads, D, k.dtype, dev, k.shape[0])
    vs = _rows(chk, "v", v, heads, D, k.dtype, dev, k.shape[0])
    chk.done()
    desc = make_paged_desc(batch, k.shape[0], heads, heads, D, num, size, columns,
                           dtype=_IO_DTYPES[k.dtype], k_stride=ks, v_stride=vs)
    _launch(dev, dsa3d_paged_append, desc, k, v, cu_q, kv_lens, pages, k_pages, v_pages)


def paged_forward(q, k_pages, v_pages, pages, kv_lens, cu_q, causal=True, scale=0.0,
                  rel_table=None, rel_buckets=None, rel_min=0, max_kv=0, need_lse=False, out=None,
                  lse=None, workspace=None):
    """Attention of the newest tokens q [rows, heads, head_dim] (packed by cu_q; one or more per
    request) over the tokens their requests hold in pages (see paged_append; the new ones' k and v
    are there already).  `max_kv`: a bound of kv_lens that the caller knows (0: what the page
    table can hold); a near one lets the work be dealt out better.  Returns (out, lse)."""
    chk = _Checks("paged_forward")
    dev = _lead_rows(chk, q)
    nq, heads, D = q.shape
    qs = _rows(chk, "q", q, heads, D, q.dtype, dev, nq)
    batch, num, size, kv_heads, kD, columns = _pages(chk, k_pages, v_pages, pages, kv_lens, cu_q,
                                                     q.dtype, dev)
    if kD != D or kv_heads < 1 or heads % kv_heads:
        chk.problems.append(f"k_pages: {kv_heads} heads x {kD} for queries of {heads} x {D}")
    lo, span, buckets = _relative(chk, rel_table, rel_buckets, rel_min, heads, dev)
    chk.optional("out", out, q.shape, q.dtype, dev)
    if need_lse:
        chk.optional("lse", lse, q.shape[:2], torch.float32, dev)
    chk.workspace(workspace, dev)
    max_kv = _int32(chk, "max_kv", max_kv)
    chk.done()
    desc = make_paged_desc(batch, nq, heads, kv_heads, D, num, size, columns, max_kv, causal,
                           _IO_DTYPES[q.dtype], scale, lo, span, buckets, qs)
    if out is None:
        out = _like(q, dev)
    if not need_lse:
        lse = None
    elif lse is None:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=dev)
    need = dsa3d_paged_forward_workspace_size(desc)
    if need and (workspace is None or workspace.numel() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _launch(dev, dsa3d_paged_forward, desc, q, k_pages, v_pages, pages, kv_lens, cu_q, rel_table,
            rel_buckets, out, lse, workspace, need)
    return out, lse
