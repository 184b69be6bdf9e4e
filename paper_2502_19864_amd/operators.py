"""The block operators on torch tensors: attention with a sliding window, sinks and a
learned relative position bias (forward and backward), and dropout.

torch supplies device memory and the stream; all compute is the library's
(ringada_attn_forward, ringada_attn_backward, ringada_dropout of include/ringada.h).
Every call is enqueued on the current stream of the tensors' device and can be
captured into a HIP graph.  Tensors of another type, device or shape than documented raise
ValueError; what the library refuses raises RingadaError.

Nothing is recorded for autograd: the backward is a call of its own, and a tensor that
requires a gradient is refused where autograd records (ValueError)."""
from __future__ import annotations

import ctypes
import functools
import struct

import torch

from . import binding as B

_DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}
# AttnDesc, AttnTensors and AttnGrads as bytes: packing them costs a fraction of building the
# ctypes structures, which is half of a small call's time on the host
_DESC, _TENSORS, _GRADS = struct.Struct("10if2i"), struct.Struct("Qqqq" * 4 + "5Q"), struct.Struct("Qqqq" * 4 + "Q")
assert (_DESC.size, _TENSORS.size, _GRADS.size) == tuple(map(ctypes.sizeof, (B.AttnDesc, B.AttnTensors, B.AttnGrads)))
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


@functools.lru_cache(maxsize=256)
def _plan(desc, with_dtable):
    """Workspace bytes (forward, backward) of a descriptor."""
    return B.ringada_attn_plan(desc, with_dtable)


def relpos_buckets(n_buckets, max_distance, bidirectional, device="cpu"):
    """The usual bucket map of a learned relative position bias (see ringada_relpos_buckets), int32
    [2 max_distance + 1], indexed by key - query + max_distance."""
    return torch.tensor(B.ringada_relpos_buckets(n_buckets, max_distance, bidirectional), dtype=torch.int32,
                        device=device)


def _on(dev, call, *args):
    """call(stream, *args) on the device's current stream, with the device made current where it is not."""
    i = dev.index
    if i == torch.cuda.current_device():
        call(_raw_stream(i), *args)
    else:
        with torch.cuda.device(dev):
            call(_raw_stream(i), *args)


def _no_graph(*tensors):
    """These calls record nothing for autograd: a tensor whose gradient it would miss is refused."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("a tensor requires a gradient: call under torch.no_grad() (as in an autograd "
                                 "Function) or on detached tensors, and take gradients from the backward calls")


def _view(name, t, shape, dtype, dev):
    if t.dtype is not dtype or t.device != dev:
        raise ValueError(f"{name}: {t.dtype} on {t.device}, q is {dtype} on {dev}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    sb, sr, sh, sd = t.stride()
    if sd != 1 and shape[3] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), sb, sr, sh


def _plain(name, t, dtype, shape, dev):
    if t is None:
        return 0
    if t.dtype is not dtype or t.device != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")
    return t.data_ptr()


def _pack(how, *values):
    try:
        return how.pack(*values)
    except struct.error as e:
        raise ValueError(f"window, sinks and scale are numbers in range: {e}") from None


def _attn(q, k, v, o, lse, causal, window, sinks, scale, len_q, len_k, table, bucket):
    """The call's desc and tensors, packed; o, lse None: allocated here (lse False: none)."""
    _no_graph(q, k, v, table)
    qs, ks, dtype, dev = q.shape, k.shape, q.dtype, q.device
    if len(qs) != 4 or len(ks) != 4:
        raise ValueError("q, k and v are [batch, rows, heads, d_head]")
    if dtype not in _DTYPES or dev.type != "cuda":
        raise ValueError(f"q: {dtype} on {dev}, expected float32 or bfloat16 on a GPU")
    (b, sq, h, dh), (kb, sk, kv, kdh) = qs, ks
    if 0 in qs or 0 in ks:
        raise ValueError("empty q or k")
    if kb != b or kdh != dh:
        raise ValueError(f"k: shape {tuple(ks)} for q of {tuple(qs)}")
    nb = r = tp = bp = 0
    if table is not None:
        if bucket is None or bucket.dim() != 1 or bucket.numel() % 2 == 0 or table.dim() != 2:
            raise ValueError("a table [n_buckets, heads] takes a bucket map [2 max_distance + 1]")
        nb, r = table.shape[0], bucket.numel() // 2
        tp = _plain("table", table, torch.float32, (nb, h), dev)
        bp = _plain("bucket", bucket, torch.int32, (2 * r + 1,), dev)
    elif bucket is not None:
        raise ValueError("a bucket map without a table")
    qv, kvw, vv = _view("q", q, qs, dtype, dev), _view("k", k, ks, dtype, dev), _view("v", v, ks, dtype, dev)
    if o is None:
        o = torch.empty(qs, dtype=dtype, device=dev)
        ov = (o.data_ptr(), sq * h * dh, h * dh, dh)
    else:
        ov = _view("o", o, qs, dtype, dev)
    if lse is None:
        lse = torch.empty((b, h, sq), dtype=torch.float32, device=dev)
        lp = lse.data_ptr()
    else:
        lp = _plain("lse", lse, torch.float32, (b, h, sq), dev) if lse is not False else 0
    desc = _pack(_DESC, _DTYPES[dtype], b, h, kv, dh, sq, sk, bool(causal), window, sinks,
                 dh ** -0.5 if scale is None else scale, nb, r)
    t = _TENSORS.pack(*qv, *kvw, *vv, *ov, lp, _plain("len_q", len_q, torch.int32, (b,), dev),
                      _plain("len_k", len_k, torch.int32, (b,), dev), tp, bp)
    return desc, t, o, lse, dev


def attention_forward(q, k, v, *, causal=False, window=0, sinks=0, scale=None, len_q=None, len_k=None, table=None,
                      bucket=None, out=None, with_lse=True):
    """q [B, Sq, H, dh], k and v [B, Sk, Hkv, dh] (any strides with dh contiguous).  Returns (o, lse):
    o as q (in `out` if given), lse [B, H, Sq] float32, which the backward takes (None
    without with_lse).  scale defaults to dh ** -0.5."""
    desc, t, o, lse, dev = _attn(q, k, v, out, None if with_lse else False, causal, window, sinks, scale, len_q, len_k,
                                 table, bucket)
    n = _plan(desc, False)[0]
    # the workspace may be freed once the call is enqueued: the allocator hands it on in stream order
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _on(dev, B.ringada_attn_forward, desc, t, ws, n)
    return o, lse if with_lse else None


def attention_backward(do, q, k, v, o, lse, *, causal=False, window=0, sinks=0, scale=None, len_q=None, len_k=None,
                       table=None, bucket=None, dtable=None, dq=None, dk=None, dv=None):
    """Gradients of attention_forward called with the same arguments.  Returns (dq, dk, dv), in the tensors
    given if any; dtable (float32, as table) is added into, and left out for a frozen table."""
    if lse is None or o is None:
        raise ValueError("the backward needs the forward's o and lse")
    desc, t, _, _, dev = _attn(q, k, v, o, lse, causal, window, sinks, scale, len_q, len_k, table, bucket)
    _no_graph(do)
    qs, ks, dtype = q.shape, k.shape, q.dtype
    if dtable is not None and table is None:
        raise ValueError("dtable without a table")
    if dq is None:
        dq = torch.empty(qs, dtype=dtype, device=dev)
    if dk is None:
        dk = torch.empty(ks, dtype=dtype, device=dev)
    if dv is None:
        dv = torch.empty(ks, dtype=dtype, device=dev)
    g = _GRADS.pack(*_view("do", do, qs, dtype, dev), *_view("dq", dq, qs, dtype, dev),
                    *_view("dk", dk, ks, dtype, dev), *_view("dv", dv, ks, dtype, dev),
                    0 if dtable is None else _plain("dtable", dtable, torch.float32, table.shape, dev))
    n = _plan(desc, dtable is not None)[1]
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _on(dev, B.ringada_attn_backward, desc, t, g, ws, n)
    return dq, dk, dv


def dropout(x, p, rng, site=0, res=None, out=None):
    """res + dropout(x) (or dropout(x) alone): the backward is the same call on the gradient.  rng: int64 [2]
    on the device, {seed, offset}; x, res and out contiguous and of one shape (out may be x or res)."""
    _no_graph(x, res)
    dtype, dev, shape = x.dtype, x.device, x.shape
    if dtype not in _DTYPES or dev.type != "cuda":
        raise ValueError(f"x: {dtype} on {dev}, expected float32 or bfloat16 on a GPU")
    xp, rp = _plain("x", x, dtype, shape, dev), _plain("res", res, dtype, shape, dev)
    gp = _plain("rng", rng, torch.int64, (2,), dev)
    y = torch.empty_like(x) if out is None else out
    yp = y.data_ptr() if out is None else _plain("out", out, dtype, shape, dev)
    _on(dev, B.ringada_dropout, _DTYPES[dtype], xp, rp or None, yp, x.numel(), p, gp, site)
    return y
