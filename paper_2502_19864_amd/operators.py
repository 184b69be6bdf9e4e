"""The block operators on torch tensors: attention with a sliding window, sinks and a
learned relative position bias (forward and backward), and dropout.

torch supplies device memory and the stream; all compute is the library's
(ringada_attn_forward, ringada_attn_backward, ringada_dropout of include/ringada.h).
Every call is enqueued on the current stream of the tensors' device and can be
captured into a HIP graph.  Tensors of another type, device or shape than documented raise
ValueError; what the library refuses raises RingadaError."""
from __future__ import annotations

import torch

from . import binding as B

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}


def relpos_buckets(n_buckets, max_distance, bidirectional, device="cpu"):
    """The usual bucket map of a learned relative position bias (see ringada_relpos_buckets), int32
    [2 max_distance + 1], indexed by key - query + max_distance."""
    return torch.tensor(B.ringada_relpos_buckets(n_buckets, max_distance, bidirectional), dtype=torch.int32,
                        device=device)


class _On:
    """The device's current stream, with the device made current for the launch where it is not."""

    def __init__(self, dev):
        self.dev, self.guard = dev, None

    def __enter__(self):
        if self.dev.index is not None and self.dev.index != torch.cuda.current_device():
            self.guard = torch.cuda.device(self.dev)
            self.guard.__enter__()
        return torch.cuda.current_stream(self.dev).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _view(name, t, shape, like):
    if t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: {t.dtype} on {t.device}, q is {like.dtype} on {like.device}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    sb, sr, sh, sd = t.stride()
    if sd != 1 and shape[3] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return B.View(t.data_ptr(), sb, sr, sh)


def _plain(name, t, dtype, shape, like):
    if t is None:
        return None
    if t.dtype != dtype or t.device != like.device or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {shape} on {like.device}")
    return t.data_ptr()


def _attn(q, k, v, o, lse, causal, window, sinks, scale, len_q, len_k, table, bucket):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v are [batch, rows, heads, d_head]")
    if q.dtype not in _DTYPES or not q.is_cuda:
        raise ValueError(f"q: {q.dtype} on {q.device}, expected float32 or bfloat16 on a GPU")
    (b, sq, h, dh), (_, sk, kv, _) = q.shape, k.shape
    if min(q.shape) < 1 or min(k.shape) < 1:
        raise ValueError("empty q or k")
    nb = r = 0
    if table is not None:
        if bucket is None or bucket.dim() != 1 or bucket.numel() % 2 == 0 or table.dim() != 2:
            raise ValueError("a table [n_buckets, heads] takes a bucket map [2 max_distance + 1]")
        nb, r = table.shape[0], bucket.numel() // 2
    desc = B.AttnDesc(_DTYPES[q.dtype], b, h, kv, dh, sq, sk, int(causal), window, sinks,
                      dh ** -0.5 if scale is None else scale, nb, r)
    cache = (b, sk, kv, dh)
    t = B.AttnTensors(_view("q", q, tuple(q.shape), q), _view("k", k, cache, q), _view("v", v, cache, q),
                      _view("o", o, tuple(q.shape), q), _plain("lse", lse, torch.float32, (b, h, sq), q),
                      _plain("len_q", len_q, torch.int32, (b,), q), _plain("len_k", len_k, torch.int32, (b,), q),
                      _plain("table", table, torch.float32, (nb, h), q),
                      None if table is None else _plain("bucket", bucket, torch.int32, (2 * r + 1,), q))
    return desc, t


def _workspace(n, like):
    return torch.empty(n, dtype=torch.uint8, device=like.device) if n else None


def attention_forward(q, k, v, *, causal=False, window=0, sinks=0, scale=None, len_q=None, len_k=None, table=None,
                      bucket=None, out=None, with_lse=True):
    """q [B, Sq, H, dh], k and v [B, Sk, Hkv, dh] (any strides with dh contiguous).  Returns (o, lse):
    o as q (in `out` if given), lse [B, H, Sq] float32, which the backward takes (None
    without with_lse).  scale defaults to dh ** -0.5."""
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device) if with_lse else None
    desc, t = _attn(q, k, v, o, lse, causal, window, sinks, scale, len_q, len_k, table, bucket)
    with _On(q.device) as stream:
        n, _ = B.ringada_attn_plan(desc, False)
        B.ringada_attn_forward(stream, desc, t, _workspace(n, q), n)
    return o, lse


def attention_backward(do, q, k, v, o, lse, *, causal=False, window=0, sinks=0, scale=None, len_q=None, len_k=None,
                       table=None, bucket=None, dtable=None, dq=None, dk=None, dv=None):
    """Gradients of attention_forward called with the same arguments.  Returns (dq, dk, dv), in the tensors
    given if any; dtable (float32, as table) is added into, and left out for a frozen table."""
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
    if lse is None:
        raise ValueError("the backward needs the forward's lse")
    desc, t = _attn(q, k, v, o, lse, causal, window, sinks, scale, len_q, len_k, table, bucket)
    sq, sk = tuple(q.shape), tuple(k.shape)
    g = B.AttnGrads(_view("do", do, sq, q), _view("dq", dq, sq, q), _view("dk", dk, sk, q), _view("dv", dv, sk, q),
                    _plain("dtable", dtable, torch.float32, (desc.n_buckets, q.shape[2]), q))
    with _On(q.device) as stream:
        _, n = B.ringada_attn_plan(desc, dtable is not None)
        B.ringada_attn_backward(stream, desc, t, g, _workspace(n, q), n)
    return dq, dk, dv


def dropout(x, p, rng, site=0, res=None, out=None):
    """res + dropout(x) (or dropout(x) alone): the backward is the same call on the gradient.  rng: int64 [2]
    on the device, {seed, offset}; x, res and out contiguous and of one shape (out may be x or res)."""
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
    if x.dtype not in _DTYPES or not x.is_cuda:
        raise ValueError(f"x: {x.dtype} on {x.device}, expected float32 or bfloat16 on a GPU")
    _plain("rng", rng, torch.int64, (2,), x)
    shape = tuple(x.shape)
    for name, t in (("x", x), ("res", res), ("out", y)):
        _plain(name, t, x.dtype, shape, x)
    with _On(x.device) as stream:
        B.ringada_dropout(stream, _DTYPES[x.dtype], x, res, y, x.numel(), p, rng, site)
    return y
