"""The block operators in float64 on the CPU, with bounds on what a kernel may be off.

The bounds count roundings.  u is half a step of the storage type (bf16 2^-8, fp32
2^-24).  A bf16 kernel rounds P and dS once (u each) on their way into a product and
each output once more; everything else is fp32, whose sums of n terms and whose scores
are off by about sqrt(n) steps of their absolute values (k32 below, eight times that):

  O:   u |O| + (u + k32) P|V|
  D:   from the stored O, off by |dO| times O's bound; from P and dP, by k32 P|dO||V|
  dS:  k32 P(|dO||V| + |D|) + P dD, and u |dS| when it enters a product
  dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO, dtable: those, times the other operand's
       absolute value, plus u of the output
"""
import math

import torch


def lens(n, seq, b):
    return [seq] * b if n is None else [min(max(int(x), 0), seq) for x in n]


def attention(q, k, v, do=None, *, causal=False, window=0, sinks=0, scale, len_q=None, len_k=None, table=None,
              bucket=None, lowp=False, d_exact=False):
    """Returns {name: (value, bound)} for o, lse and, with do, dq, dk, dv, dtable.  lowp: bf16 storage;
    d_exact: D formed from P and dP.  Rows past the lengths may hold anything."""
    q, k, v = (x.detach().double().cpu() for x in (q, k, v))
    B, Sq, H, dh = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    g, u = H // Hkv, 2.0 ** -8 if lowp else 2.0 ** -24
    up = u if lowp else 0.0  # of P and dS on their way into a product
    out = {n: [torch.zeros_like(x), torch.zeros_like(x)] for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    out["lse"] = [torch.full((B, H, Sq), -math.inf, dtype=torch.float64), torch.zeros(B, H, Sq, dtype=torch.float64)]
    if table is not None:
        table, bucket = table.detach().double().cpu(), bucket.cpu().long().clamp(0, table.shape[0] - 1)
        R = bucket.numel() // 2
        out["dtable"] = [torch.zeros_like(table), torch.zeros_like(table)]
    for b, (lq, lk) in enumerate(zip(lens(len_q, Sq, B), lens(len_k, Sk, B))):
        if not lq or not lk:
            continue
        p_ = torch.arange(lq)[:, None] + (lk - lq)
        j = torch.arange(lk)[None, :]
        vis = torch.ones(lq, lk, dtype=torch.bool)
        if causal:
            vis &= j <= p_
        if window:
            vis &= ((p_ - j).abs() < window) | (j < sinks)
        for h in range(H):
            Q, K, V = q[b, :lq, h], k[b, :lk, h // g], v[b, :lk, h // g]
            x = Q @ K.T * scale
            ok = vis
            if table is not None:
                at = bucket[(j - p_).clamp(-R, R) + R]
                bias = table[at, h]
                ok = vis & (bias > -1e30)
                x = x + bias.clamp(min=-1e30)
            x = x.masked_fill(~ok, -math.inf)
            m = x.amax(1, keepdim=True)
            m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
            e = torch.exp(x - m)
            s = e.sum(1, keepdim=True)
            P = e / torch.where(s == 0, torch.ones_like(s), s)
            big = float((scale * (Q.abs() @ K.abs().T)).max() + (bias[ok].abs().max() if table is not None and ok.any() else 0))
            k32 = 2.0 ** -24 * 8 * math.sqrt(dh + lk + lq) * (1 + big)
            O, A = P @ V, P @ V.abs()
            bo = u * O.abs() + (up + k32) * A
            out["o"][0][b, :lq, h], out["o"][1][b, :lq, h] = O, bo
            seen = s[:, 0] > 0
            out["lse"][0][b, h, :lq] = torch.where(seen, (m + torch.log(s))[:, 0] / math.log(2), -math.inf)
            out["lse"][1][b, h, :lq] = k32 + 2.0 ** -22 * big
            if do is None:
                continue
            dO = do[b, :lq, h].detach().double().cpu()
            dP, dA = dO @ V.T, dO.abs() @ V.abs().T
            D = (P * dP).sum(1, keepdim=True)
            dD = (dO.abs() * (k32 * A if d_exact else bo)).sum(1, keepdim=True)
            dS = P * (dP - D)
            bs = k32 * P * (dA + (P * dA).sum(1, keepdim=True)) + P * dD
            es = up * (dS.abs() + bs) + bs
            for n, val, bound in (("dq", scale * dS @ K, scale * es @ K.abs()),):
                out[n][0][b, :lq, h], out[n][1][b, :lq, h] = val, bound
            out["dk"][0][b, :lk, h // g] += scale * dS.T @ Q
            out["dk"][1][b, :lk, h // g] += scale * es.T @ Q.abs()
            out["dv"][0][b, :lk, h // g] += P.T @ dO
            out["dv"][1][b, :lk, h // g] += (up + k32) * (P.T @ dO.abs())
            if table is not None:
                out["dtable"][0][:, h].index_add_(0, at.reshape(-1), dS.reshape(-1))
                out["dtable"][1][:, h].index_add_(0, at.reshape(-1), bs.reshape(-1))
    for n in ("dq", "dk", "dv", "dtable"):
        if n in out:
            out[n][1] = out[n][1] * 1.01 + (2.0 ** -24 if n == "dtable" else u) * (out[n][0].abs() + out[n][1])
    out["o"][1] *= 1.01
    if do is None:
        out = {n: out[n] for n in ("o", "lse")}
    return {n: tuple(x) for n, x in out.items()}


def check(name, got, want, bound, least=1e-30):
    """|got - want| <= bound element by element (0 allowed where nothing was computed)."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{name}: infinities differ"
    off = torch.where(inf, torch.zeros_like(want), (got - torch.where(inf, torch.zeros_like(want), want)).abs())
    off = torch.where(inf, torch.zeros_like(off), off)
    assert not torch.isnan(off).any(), f"{name}: NaN"
    ratio = (off / (bound + least)).max().item() if off.numel() else 0.0
    assert ratio <= 1.0, f"{name}: off by {ratio:.3f} of its bound"
    return ratio


def philox(n, seed, offset, site):
    """The 16 random bits of each of n elements, in Python integers."""
    out = []
    for c in range((n + 7) // 8):
        x, k = [c & 0xFFFFFFFF, site, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
            x = [(b >> 32) ^ x[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ x[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out += [h for w in x for h in (w & 0xFFFF, w >> 16)]
    return out[:n]
