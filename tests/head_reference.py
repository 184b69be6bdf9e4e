"""Norms, the rotary embedding and the vocabulary head in float64, with bounds on what a kernel
may be off.

The bounds count roundings.  u is half a step of the storage type (bf16 2^-8, fp32
2^-24), e = 2^-24 that of the fp32 arithmetic.  A sum of n fp32 terms held by many threads is off by at most (steps in a
row) e of the terms' absolute values: 64 where a row is summed (32 in a thread, then a tree), rows / groups +
groups / 32 + 64 for the sums over rows; a matrix product of n terms by about 8 sqrt(n) e of them.
"""
import math

import torch

E = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def norm(s, gain, shift, rms, eps, dy=None, dskip=None, groups=512):
    """{name: (value, bound)} of y and with dy of dx, dgain, dshift; s [rows, d] as stored."""
    u, k = half_step(s.dtype), 64 * E
    x, g = s.double(), gain.double()
    mean = torch.zeros_like(x[:, :1]) if rms else x.mean(1, keepdim=True)
    size = x.abs() + (0 if rms else x.abs().mean(1, keepdim=True))
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    xh = (x - mean) * rstd
    # the mean's error enters the variance in its square and times the mean of x - mean, which is none
    exh = k * (rstd * size + xh.abs())
    y = xh * g + (0 if shift is None else shift.double())
    out = {"y": (y, 1.01 * (exh * g.abs() + 2 * E * ((xh * g).abs() + y.abs())) + u * y.abs() * 1.01)}
    if dy is None:
        return out
    d = dy.double()
    a = d * g
    m2, m2a = (a * xh).mean(1, keepdim=True), (a * xh).abs().mean(1, keepdim=True)
    em2 = k * m2a + (a.abs() * exh).mean(1, keepdim=True)
    m1 = torch.zeros_like(m2) if rms else a.mean(1, keepdim=True)
    em1 = torch.zeros_like(m2) if rms else k * a.abs().mean(1, keepdim=True)
    inner = a - m1 - xh * m2
    dx = inner * rstd
    # 4 roundings on the way, and rstd's own relative error (k)
    e = rstd * (em1 + em2 * xh.abs() + exh * m2.abs() + 4 * E * (a.abs() + m1.abs() + (xh * m2).abs())) + k * dx.abs()
    if dskip is not None:
        dx = dx + dskip.double()
        e = e + 2 * E * dx.abs()
    out["dx"] = (dx, 1.01 * e + u * dx.abs() * 1.01)
    rows = s.shape[0]
    kr = (rows / max(1, min(rows, groups)) + groups / 32 + 64) * E
    out["dgain"] = ((d * xh).sum(0), (kr * (d * xh).abs() + d.abs() * exh).sum(0) * 1.01)
    out["dshift"] = (d.sum(0), kr * d.abs().sum(0) * 1.01)
    return out


def rotary(x, positions, freq, sections, inverse=False):
    """(value, bound).  positions [axes, B, S].  An angle's place in the turn is rounded once (3.2 e), sine and cosine are good to
    2 steps; then three roundings of the products and the sum, and the storage's."""
    p = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    angle = positions.double()[axis].permute(1, 2, 0) * freq.double()
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None] * (-1 if inverse else 1)
    d = x.double()
    a, b, rest = d[..., :p], d[..., p:2 * p], d[..., 2 * p:]
    out = torch.cat((a * c - b * s, b * c + a * s, rest), -1)
    size = torch.cat((a.abs() + b.abs(), a.abs() + b.abs(), torch.zeros_like(rest)), -1)
    return out, 10 * E * size + half_step(x.dtype) * out.abs() * 1.01


def vocab(h, w, labels, dloss=None):
    """{name: (value, bound)} of loss, lse and with dloss of dh, dw.  Rows that do not count may hold anything."""
    u = half_step(h.dtype)
    up = u if h.dtype is torch.bfloat16 else 0.0  # of P on its way into a product
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    at = ((labels >= 0) & (labels < V)).nonzero()[:, 0]
    up = up * up if at.numel() <= 64 else up  # two parts
    H, W, lab = h[at].double(), w.double(), labels[at].long()[:, None]
    s, A = H @ W.T, H.abs() @ W.abs().T
    es = 8 * math.sqrt(d) * E * A
    lse = torch.logsumexp(s, 1, keepdim=True) if at.numel() else s[:, :1]
    logp = s - lse
    p = logp.exp()
    # exp: its argument's rounding and the function's two steps; log: a rounding of lse
    elog = es + (p * (es + 4 * E * (1 - logp))).sum(1, keepdim=True) + 4 * E * (1 + (s.amax(1, keepdim=True) - lse).abs() if at.numel() else 0)
    loss = -logp.gather(1, lab)
    eloss = elog.gather(1, lab) + 4 * E * loss.abs()
    z = lambda *sh: torch.zeros(*sh, dtype=torch.float64, device=h.device)
    full = lambda v: z(n, *v.shape[1:]).index_copy_(0, at, v)
    out = {"loss": (full(loss)[:, 0], full(eloss)[:, 0]),
           "lse": (full(lse)[:, 0], full((elog - es).amax(1, keepdim=True) + es.gather(1, s.argmax(1, keepdim=True)) + 4 * E * lse.abs())[:, 0]
                   if at.numel() else z(n))}
    if dloss is None:
        return out
    g = dloss[at].double()[:, None]
    P = p.scatter(1, lab, torch.expm1(-loss))
    # with bf16 tensors a logit is held in fp16 as its distance to the largest near it, which is no more than that to lse: half a
    # step of it, 2^-11 (2^-25 near zero)
    e16 = 2.0 ** -11 * logp.abs() + 2.0 ** -24 if up else 0.0
    eP = (p * (elog + e16 + 4 * E * (1 + logp.abs()))).scatter(1, lab, p.gather(1, lab) * eloss + 4 * E * P.gather(1, lab).abs())
    P, eP = g * P, g.abs() * eP
    eP = eP + up * (P.abs() + eP) * 1.01
    kv, kn = 8 * math.sqrt(V) * E, 8 * math.sqrt(max(1, at.numel())) * E
    dh = P @ W
    eh = (eP + kv * P.abs()) @ W.abs()
    dw = P.T @ H
    ew = (eP + kn * P.abs()).T @ H.abs()
    out["dh"] = (full(dh), full(1.01 * eh + u * (dh.abs() + eh) * 1.01))
    out["dw"] = (dw, 1.01 * ew + u * (dw.abs() + ew) * 1.01)
    return out


def check(name, got, want, bound, least=1e-37):
    """|got - want| <= bound element by element (least: what underflows)."""
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs()
    assert not torch.isnan(off).any(), f"{name}: NaN"
    ratio = (off / (bound + least)).max().item() if off.numel() else 0.0
    assert ratio <= 1.0, f"{name}: off by {ratio:.3f} of its bound"
    return ratio
