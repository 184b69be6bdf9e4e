"""The block operators on torch tensors: attention with a sliding window, sinks and a
learned relative position bias (forward and backward), dropout, LayerNorm and RMSNorm with
their gradients, the rotary embedding, and a vocabulary head with softmax cross entropy.

torch supplies device memory and the stream; all compute is the library's
(the block operators of include/ringada.h).
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
_ROWS, _NORM, _ROTARY, _VOCAB = struct.Struct("Qq"), struct.Struct("2iqif"), struct.Struct("12i"), struct.Struct("4i")
_VOCAB_TENSORS, _VIEW = struct.Struct("QqQq4QQqQq"), struct.Struct("Qqqq")
assert (_ROWS.size, _NORM.size, _ROTARY.size, _VOCAB.size, _VOCAB_TENSORS.size, _VIEW.size) == tuple(
    map(ctypes.sizeof, (B.Rows, B.NormDesc, B.RotaryDesc, B.VocabDesc, B.VocabTensors, B.View)))
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
        raise ValueError(f"window, sinks, scale, eps and sections are numbers in range: {e}") from None


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


# ---------------------------------------------------------------- rows of d elements: norms and the vocabulary head
def _fresh(t):
    """A new contiguous tensor as t (the quickest of torch's ways: a small call is bound by its time on the host)."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def _storage(name, t):
    if t.dtype not in _DTYPES or t.device.type != "cuda":
        raise ValueError(f"{name}: {t.dtype} on {t.device}, expected float32 or bfloat16 on a GPU")
    if t.numel() == 0 or t.dim() < 1:
        raise ValueError(f"{name}: shape {tuple(t.shape)} is empty")
    return t.dtype, t.device


def _rows(name, t, shape, dtype, dev):
    """(address, row stride) of a tensor [..., d]: any row stride in two dimensions, else contiguous."""
    if t.dtype is not dtype or t.device != dev or t.shape != shape:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtype} {tuple(shape)} on {dev}")
    d = shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), d
    if t.dim() != 2 or (t.stride(1) != 1 and d != 1):
        raise ValueError(f"{name}: rows must be contiguous, and evenly spaced in more than two dimensions")
    return t.data_ptr(), t.stride(0)


def _out_rows(name, t, like, shape, dtype, dev):
    """An output and its packed rows: t, or a new tensor."""
    if t is None:
        t = _fresh(like)
        return t, _ROWS.pack(t.data_ptr(), shape[-1])
    return t, _ROWS.pack(*_rows(name, t, shape, dtype, dev))


@functools.lru_cache(maxsize=256)
def _norm_plan(desc):
    return B.ringada_norm_plan(desc)


def _norm_desc(x, rms, eps):
    d = x.shape[-1]
    return _pack(_NORM, _DTYPES[x.dtype], B.NORM_RMS if rms else B.NORM_LAYER, x.numel() // d, d, eps)


def norm_forward(x, gain, shift=None, *, rms=False, eps=1e-5, res=None, out=None, out_sum=None, with_stats=True):
    """LayerNorm (RMSNorm with rms) of x + res over the last dimension: x and res [..., d], gain and shift [d] of
    x's type.  Returns (y, s, stats): y as x (in `out` if given), s = x + res as stored (in `out_sum` if given; x itself
    without res), stats [rows, 2] float32 for the backward (None without with_stats).  out and out_sum may
    be x or res."""
    _no_graph(x, gain, shift, res)
    dtype, dev = _storage("x", x)
    shape, d = x.shape, x.shape[-1]
    desc = _norm_desc(x, rms, eps)
    if res is None and out_sum is not None:
        raise ValueError("out_sum without res")
    xr = _ROWS.pack(*_rows("x", x, shape, dtype, dev))
    rr = sr = None
    s = x
    if res is not None:
        rr = _ROWS.pack(*_rows("res", res, shape, dtype, dev))
        s, sr = _out_rows("out_sum", out_sum, x, shape, dtype, dev)
    y, yr = _out_rows("out", out, x, shape, dtype, dev)
    gp, bp = _plain("gain", gain, dtype, (d,), dev), _plain("shift", shift, dtype, (d,), dev)
    stats = torch.empty((x.numel() // d, 2), dtype=torch.float32, device=dev) if with_stats else None
    _on(dev, B.ringada_norm_forward, desc, xr, rr, sr, gp, bp or None, yr, stats)
    return y, s, stats


def norm_backward(dy, s, gain, stats, *, rms=False, dskip=None, dgain=None, dshift=None, out=None):
    """The gradient of norm_forward's s (of x, and of res): the norm's from dy, plus dskip, what reaches s past it.  dgain
    and dshift (float32 [d]) are added into, and left out for frozen ones.  Returns dx (in `out` if given, which may be dy, dskip or
    s)."""
    _no_graph(dy, s, gain, dskip)
    dtype, dev = _storage("s", s)
    shape, d = s.shape, s.shape[-1]
    desc = _norm_desc(s, rms, 0.0)
    rows = s.numel() // d
    if stats is None:
        raise ValueError("the backward needs the forward's stats")
    dx, xr = _out_rows("out", out, s, shape, dtype, dev)
    dyr, sr = _ROWS.pack(*_rows("dy", dy, shape, dtype, dev)), _ROWS.pack(*_rows("s", s, shape, dtype, dev))
    kr = None if dskip is None else _ROWS.pack(*_rows("dskip", dskip, shape, dtype, dev))
    gp, tp = _plain("gain", gain, dtype, (d,), dev), _plain("stats", stats, torch.float32, (rows, 2), dev)
    dgp, dbp = _plain("dgain", dgain, torch.float32, (d,), dev), _plain("dshift", dshift, torch.float32, (d,), dev)
    n = _norm_plan(desc) if dgp or dbp else 0
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _on(dev, B.ringada_norm_backward, desc, dyr, kr, sr, gp, tp, xr, dgp or None, dbp or None, ws, n)
    return dx


def _out_view(name, t, like, shape, dtype, dev):
    """As _out_rows, of [batch, rows, heads, d_head]."""
    if t is None:
        t = _fresh(like)
        _, rows, h, dh = shape
        return t, _VIEW.pack(t.data_ptr(), rows * h * dh, h * dh, dh)
    return t, _VIEW.pack(*_view(name, t, shape, dtype, dev))


def rotary_frequencies(sections, theta=10000.0, shared=False, device="cpu"):
    """The usual frequencies (see ringada_rotary_frequencies), float64 [sum(sections)]."""
    return torch.tensor(B.ringada_rotary_frequencies(tuple(sections), theta, shared), dtype=torch.float64, device=device)


def rotary(q, k=None, *, positions, freq, sections=None, inverse=False, out_q=None, out_k=None):
    """q [B, S, H, dh] and k [B, S, Hkv, dh] (any strides with dh contiguous) turned by their positions: int32
    [axes, B, S], or [B, S] for one axis, contiguous.  freq: float64, the angle of each pair per position; sections:
    the pairs of each axis (default: one axis has them all).  inverse turns back, which is the backward.  Returns
    (q, k) turned (k None without k), in out_q and out_k if given, which may be q and k themselves."""
    _no_graph(q, k, freq)
    dtype, dev = _storage("q", q)
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q and k are [batch, rows, heads, d_head]")
    if k is None and out_k is not None:
        raise ValueError("out_k without k")
    b, rows, h, dh = q.shape
    sections = (freq.numel(),) if sections is None else tuple(sections)
    axes = len(sections)
    if not 1 <= axes <= 4:
        raise ValueError("sections: one to four axes")
    pshape = (b, rows) if axes == 1 and positions.dim() == 2 else (axes, b, rows)
    pp = _plain("positions", positions, torch.int32, pshape, dev)
    fp = _plain("freq", freq, torch.float64, (sum(sections),), dev)
    kv = 0
    kr = okr = None
    if k is not None:
        kv = k.shape[2]
        kshape = (b, rows, kv, dh)
        if kv == 0:
            raise ValueError("k: no heads")
        kr = _VIEW.pack(*_view("k", k, kshape, dtype, dev))
        ok, okr = _out_view("out_k", out_k, k, kshape, dtype, dev)
    oq, oqr = _out_view("out_q", out_q, q, (b, rows, h, dh), dtype, dev)
    desc = _pack(_ROTARY, _DTYPES[dtype], b, rows, h, kv, dh, axes, *sections, *([0] * (4 - axes)), bool(inverse))
    _on(dev, B.ringada_rotary, desc, _VIEW.pack(*_view("q", q, q.shape, dtype, dev)), kr, pp, fp, oqr, okr)
    return oq, (ok if k is not None else None)


@functools.lru_cache(maxsize=256)
def _vocab_plan(desc):
    return B.ringada_vocab_plan(desc)


def _vocab(h, w):
    _no_graph(h, w)
    dtype, dev = _storage("h", h)
    if w.dim() != 2 or w.shape[1] != h.shape[-1]:
        raise ValueError(f"w: shape {tuple(w.shape)}, expected [vocab, {h.shape[-1]}]")
    if w.shape[0] == 0:
        raise ValueError("w: no classes")
    n, d = h.numel() // h.shape[-1], h.shape[-1]
    desc = _pack(_VOCAB, _DTYPES[dtype], n, d, w.shape[0])
    return desc, _rows("h", h, h.shape, dtype, dev), _rows("w", w, w.shape, dtype, dev), n, dtype, dev


def _vocab_ce(h, w, labels, dloss, dh, dw):
    desc, hr, wr, n, dtype, dev = _vocab(h, w)
    _no_graph(dloss)
    lead = h.shape[:-1]
    lp, gp = _plain("labels", labels, torch.int32, lead, dev), _plain("dloss", dloss, torch.float32, lead, dev)
    loss, lse = torch.empty((2,) + lead, dtype=torch.float32, device=dev)
    dhr = (0, 0) if dh is None else _rows("dh", dh, h.shape, dtype, dev)
    dwr = (0, 0) if dw is None else _rows("dw", dw, w.shape, dtype, dev)
    t = _VOCAB_TENSORS.pack(*hr, *wr, lp, loss.data_ptr(), lse.data_ptr(), gp, *dhr, *dwr)
    size = _vocab_plan(desc)[0 if dloss is None else 1]
    ws = torch.empty(size, dtype=torch.uint8, device=dev)
    _on(dev, B.ringada_vocab_ce, desc, t, ws, size)
    return loss, lse


def vocab_ce_forward(h, w, labels):
    """Softmax cross entropy of the logits h w^T: h [..., d], w [vocab, d], labels int32 [...]; a label outside
    [0, vocab) is of a row that does not count.  Returns (loss, lse), float32 [...], 0 for such rows."""
    return _vocab_ce(h, w, labels, None, None, None)


def vocab_ce_train(h, w, labels, dloss, *, frozen=False, dh=None, dw=None):
    """vocab_ce_forward and the gradients in one call; dloss float32 [...]: the gradient that arrives at each row's loss (for
    a mean over the rows that count, one over their number).  Returns (loss, lse, dh, dw), gradients as h
    and w (in the tensors given if any); frozen: the head is not trained, dw is None."""
    if dloss is None:
        raise ValueError("gradients need dloss")
    if frozen and dw is not None:
        raise ValueError("dw of a frozen head")
    if dh is None:
        dh = _fresh(h)
    if dw is None and not frozen:
        dw = _fresh(w)
    loss, lse = _vocab_ce(h, w, labels, dloss, dh, dw)
    return loss, lse, dh, dw


def vocab_next(h, w):
    """The likeliest class of every row of h [..., d] under w [vocab, d] (the lowest of equal ones), int32 [...], and
    its log-probability, float32 [...]."""
    desc, hr, wr, n, dtype, dev = _vocab(h, w)
    token = torch.empty(h.shape[:-1], dtype=torch.int32, device=dev)
    logprob = torch.empty(h.shape[:-1], dtype=torch.float32, device=dev)
    size = _vocab_plan(desc)[2]
    ws = torch.empty(size, dtype=torch.uint8, device=dev)
    _on(dev, B.ringada_vocab_next, desc, _ROWS.pack(*hr), _ROWS.pack(*wr), token, logprob, ws, size)
    return token, logprob
