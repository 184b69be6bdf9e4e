"""The operators between a block's attention and the loss, as calls of their own: a
vocabulary head with softmax cross entropy and its gradients, the next token from
the same head, LayerNorm / RMSNorm with a residual and the gradients of gain and
shift, and the rotary embedding over one or several axes.

A case is one pass through one operator:

* "ce_score":   loss and log-sum-exp of every row (forward);
* "ce_train":   those and the gradients of the hidden states and, unless frozen, of the head;
* "next":       the likeliest token of every row and its log-probability;
* "norm":       y = norm(x [+ res]) (forward);
* "norm_train": forward and backward, the gradients of gain and shift included;
* "rotary":     q and k turned by their positions;
* "rotary_train": that and its backward, the turn back of the gradients.

run() computes the operators in plain torch, in 32 bits, or with `own` through
the library's calls.

Vocabulary head: s = h w^T over w [vocab, d]; a row with a label outside [0, vocab)
does not count: loss 0, log-sum-exp 0, no gradient.  Of the others loss = lse - s[label],
and with g the gradient that arrives at the row's loss P = g (softmax(s) - onehot),
dh = P w, dw = P^T h.

Norm: s = x + res in the storage type, y = (s - mean) / sqrt(var + eps) gain + shift
(LayerNorm), or s / sqrt(mean(s^2) + eps) gain (RMSNorm).  The backward adds dskip, the
gradient that reaches s past the norm.

Rotary: pairs (i, i + P) of a head, P the number of pairs, turn by position[axis of i] *
freq[i]; dimensions from 2 P on stay.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5


# ---------------------------------------------------------------- cases
def _ce(name, kind, n, d, vocab, counted=1.0, frozen=False, dtype="bf16"):
    case = dict(kind=kind, dtype=dtype, n=n, d=d, vocab=vocab, counted=counted, frozen=frozen)
    return dict(case, name=name) if name else case


def _norm(name, kind, rows, d, rms, res, shift, dtype="bf16"):
    case = dict(kind=kind, dtype=dtype, rows=rows, d=d, rms=rms, res=res, shift=shift)
    return dict(case, name=name) if name else case


def _rotary(name, kind, batch, rows, heads, kv_heads, dh, sections, first, shared=False, dtype="bf16"):
    """sections: pairs of each axis, as "64" or "16+24+24"; first: the position that sequences start near."""
    case = dict(kind=kind, dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dh=dh,
                sections=sections, first=first, shared=shared)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the small fp32 stage with a vocabulary of its own: launches, little work
        _ce("ce_tiny_f32", "ce_train", 4 * 32, 128, 512, dtype="f32"),
        # a BERT-base batch in masked-token training: 15 % of the positions have a label
        _ce("ce_bert_masked", "ce_train", 32 * 128, 768, 30011, counted=0.15),
        # the 7B share's batch, every position predicts its next token, head trained
        _ce("ce_llama", "ce_train", 4 * 512, 4096, 32000),
        # a long batch over a large vocabulary, head frozen (adapters alone are trained), some padding
        _ce("ce_frozen_large", "ce_train", 8192, 4096, 65537, counted=0.9, frozen=True),
        # the log-probabilities of a short answer's tokens
        _ce("score_short", "ce_score", 333, 4096, 32000),
        # the next token of one conversation, and of a few over a large vocabulary
        _ce("next_one", "next", 1, 4096, 32000),
        _ce("next_few", "next", 5, 2048, 131071),
        # a decoded token's norm behind the residual
        _norm("norm_decode", "norm", 1, 4096, True, True, False),
        # a BERT-base sublayer's norm in training, post-LN
        _norm("norm_bert_train", "norm_train", 32 * 128, 768, False, True, True),
        # a long batch at the 7B width, pre-RMSNorm in training
        _norm("norm_llama_train", "norm_train", 8 * 2048, 4096, True, True, False),
        # a new token of each of three conversations, far along
        _rotary("rotary_decode", "rotary", 3, 1, 32, 8, 128, "64", 100000),
        # clips of odd length in training: time, height and width turn parts of a head
        _rotary("rotary_video_train", "rotary_train", 2, 4097, 16, 16, 128, "16+24+24", 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_LOGITS, MOST_PRODUCT = 8192 * 65537, 8192 * 65537 * 4096  # of the largest listed case


def draw(rng):
    while True:
        kind = rng.choice(("ce_train", "ce_train", "ce_train", "ce_score", "next", "norm", "norm_train", "norm_train",
                           "rotary", "rotary_train"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        if kind in ("ce_train", "ce_score", "next"):
            d = _log(rng, 8, 4096)
            if dtype == "bf16":
                d = max(8, d // 8 * 8)
            n = _log(rng, 1, 32) if kind == "next" else _log(rng, 1, 16384)
            vocab = _log(rng, 40, 160000)
            if n * vocab > MOST_LOGITS or n * vocab * d > MOST_PRODUCT / (16 if dtype == "f32" else 1.5):
                continue
            counted = 1.0 if kind == "next" else rng.choice((1.0, 1.0, 0.9, 0.5, 0.15))
            return _ce(None, kind, n, d, vocab, counted, kind == "ce_train" and rng.random() < 0.3, dtype)
        if kind in ("norm", "norm_train"):
            d, rows = _log(rng, 16, 8192), _log(rng, 1, 65536)
            if rng.random() < 0.6:
                d = max(16, d // 8 * 8)
            if d * rows > 1 << 27:
                continue
            rms = rng.random() < 0.5
            return _norm(None, kind, rows, d, rms, rng.random() < 0.5, not rms and rng.random() < 0.8, dtype)
        kv = rng.choice((1, 2, 4, 8, 12, 16))
        heads = kv * rng.choice((1, 1, 2, 4))
        dh = rng.choice((32, 64, 64, 80, 96, 128, 128, 256))
        batch, rows = _log(rng, 1, 16), 1 if kind == "rotary" and rng.random() < 0.4 else _log(rng, 2, 16384)
        if batch * rows * (heads + kv) * dh > 1 << 26:
            continue
        p = dh // 2
        sections = rng.choice((str(p), str(p), str(p // 2), f"{p // 4}+{p - p // 4}", f"{p // 4}+{p // 2}+{p // 4}"))
        return _rotary(None, kind, batch, rows, heads, kv, dh, sections, rng.choice((0, 0, 1000, 1 << 20)),
                       rng.random() < 0.5, dtype)


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(shape, generator=g, device=DEV) * std + mean).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    if case["kind"] in ("ce_train", "ce_score", "next"):
        n, d, vocab = case["n"], case["d"], case["vocab"]
        w = normal(vocab, d, std=d ** -0.5)
        labels = (uniform(n) * vocab).int().clamp(max=vocab - 1)
        # what a model has learnt: hidden states lean to their label's row, some little and some much
        h = (torch.randn((n, d), generator=g, device=DEV) + 12 * uniform(n, 1) * w[labels.long()].float()).to(dt)
        st = dict(case=case, h=h, w=w)
        if case["kind"] == "next":
            return st
        keep = uniform(n) < case["counted"]
        keep[0] |= n < 8  # a short batch has a row that counts
        st["labels"] = torch.where(keep, labels, torch.full_like(labels, -1))
        if case["kind"] == "ce_train":
            st["dloss"] = torch.where(keep, 1.0 / keep.sum().clamp(min=1), 0.0).float()
        return st
    if case["kind"] in ("norm", "norm_train"):
        rows, d = case["rows"], case["d"]
        loud = torch.where(uniform(d) < 0.01, 20.0, 1.0)  # a few channels of a residual stream are loud
        st = dict(case=case, x=((torch.randn((rows, d), generator=g, device=DEV) + 0.3) * loud).to(dt),
                  gain=normal(d, std=0.2, mean=1.0), shift=normal(d, std=0.2) if case["shift"] else None,
                  res=normal(rows, d) if case["res"] else None)
        if case["kind"] == "norm_train":
            st["dy"] = normal(rows, d, std=1e-2)
            st["dskip"] = normal(rows, d, std=1e-2) if case["res"] else None
        return st
    b, rows, h, kv, dh = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "dh"))
    sections = _sections(case)
    qkv = normal(b, rows, h + 2 * kv, dh)  # one projection wrote Q, K and V side by side
    st = dict(case=case, q=qkv[:, :, :h], k=qkv[:, :, h:h + kv], freq=torch.tensor(_frequencies(case), dtype=torch.float64,
                                                                                   device=DEV))
    start = (uniform(b, 1) * 512).int() + case["first"]
    step = torch.arange(rows, device=DEV, dtype=torch.int32)[None].expand(b, rows)
    if len(sections) == 1:
        axes = [start + step]
    else:  # frames of at most 24 x 32 patches, row by row
        axes = [start + step // 768, step // 32 % 24, step % 32][-len(sections):]
        axes[0] = axes[0] + start
    st["positions"] = torch.stack([a.expand(b, rows) for a in axes]).int().contiguous()
    if case["kind"] == "rotary_train":
        st["dq"], st["dk"] = normal(b, rows, h, dh, std=1e-2), normal(b, rows, kv, dh, std=1e-2)
    return st


def _sections(case):
    return tuple(int(x) for x in case["sections"].split("+"))


def _frequencies(case):
    """The pairs' angles per position: 10000^(-j / m) for the j-th of the m pairs of an axis, or of all pairs (shared)."""
    sections = _sections(case)
    if case["shared"]:
        sections = (sum(sections),)
    return [10000.0 ** (-j / m) for m in sections for j in range(m)]


# ---------------------------------------------------------------- the plain forms
def _plain_ce(st, train):
    c, dt = st["case"], st["h"].dtype
    n, d, vocab = c["n"], c["d"], c["vocab"]
    at = ((st["labels"] >= 0) & (st["labels"] < vocab)).nonzero()[:, 0]  # the rows that count, as a user picks them
    label = st["labels"][at].long()[:, None]
    h, w = st["h"][at].float(), st["w"].float()
    s = torch.matmul(h, w.t())
    m = s.amax(1, keepdim=True) if at.numel() else s[:, :1]
    target = s.gather(1, label)
    p = (s - m).exp_()
    z = p.sum(1, keepdim=True)
    lse = m + z.log()
    out = dict(loss=torch.zeros(n, device=DEV).index_copy_(0, at, (lse - target)[:, 0]),
               lse=torch.zeros(n, device=DEV).index_copy_(0, at, lse[:, 0]))
    if train:
        g = st["dloss"][at][:, None]
        p *= g / z
        p.scatter_(1, label, g * torch.expm1(target - lse))  # P - 1 without losing what is small of it
        out["dh"] = torch.zeros(n, d, dtype=dt, device=DEV).index_copy_(0, at, torch.matmul(p, w).to(dt))
        if not c["frozen"]:
            out["dw"] = torch.matmul(p.t(), h).to(dt)
    return out


def _plain_next(st):
    s = torch.matmul(st["h"].float(), st["w"].float().t())
    m = s.amax(1, keepdim=True)
    j = torch.arange(s.shape[1], device=DEV)[None]
    token = torch.where(s == m, j, s.shape[1]).amin(1).int()  # the lowest of equal ones
    return dict(token=token, logprob=-(s - m).exp_().sum(1).log())


def _plain_norm(st, train):
    c, dt = st["case"], st["x"].dtype
    s = st["x"]
    if st["res"] is not None:
        s = (s.float() + st["res"].float()).to(dt)
    f, gain = s.float(), st["gain"].float()
    if not c["rms"]:
        f = f - f.mean(1, keepdim=True)
    rstd = (f.square().mean(1, keepdim=True) + EPS).rsqrt()
    xh = f * rstd
    y = xh * gain
    if st["shift"] is not None:
        y = y + st["shift"].float()
    out = dict(y=y.to(dt))
    if st["res"] is not None:
        out["s"] = s
    if train:
        dy = st["dy"].float()
        a = dy * gain
        dx = a - xh * (a * xh).mean(1, keepdim=True)
        if not c["rms"]:
            dx = dx - a.mean(1, keepdim=True)
        dx = dx * rstd
        if st["dskip"] is not None:
            dx = dx + st["dskip"].float()
        out["dx"] = dx.to(dt)
        out["dgain"] = (dy * xh).sum(0)
        if st["shift"] is not None:
            out["dshift"] = dy.sum(0)
    return out


def _plain_rotary(st, names, back):
    c = st["case"]
    sections = _sections(c)
    p = sum(sections)
    axis = torch.repeat_interleave(torch.arange(len(sections), device=DEV), torch.tensor(sections, device=DEV),
                                   output_size=p)
    angle = st["positions"].double()[axis].permute(1, 2, 0) * st["freq"]  # far positions need 64 bits
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    if back:
        sin = -sin
    out = {}
    for name in names:
        x = st[name].float()
        a, b, rest = x[..., :p], x[..., p:2 * p], x[..., 2 * p:]
        out[name + "_turned"] = torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1).to(st[name].dtype)
    return out


# ---------------------------------------------------------------- a pass
def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        if kind == "next":
            return _plain_next(state)
        if kind.startswith("ce"):
            return _plain_ce(state, kind == "ce_train")
        if kind.startswith("norm"):
            return _plain_norm(state, kind == "norm_train")
        out = _plain_rotary(state, ("q", "k"), False)
        if kind == "rotary_train":
            out.update(_plain_rotary(state, ("dq", "dk"), True))
        return out
    from paper_2502_19864_amd import operators as ops
    if kind == "next":
        token, logprob = ops.vocab_next(state["h"], state["w"])
        return dict(token=token, logprob=logprob)
    if kind == "ce_score":
        loss, lse = ops.vocab_ce_forward(state["h"], state["w"], state["labels"])
        return dict(loss=loss, lse=lse)
    if kind == "ce_train":
        loss, lse, dh, dw = ops.vocab_ce_train(state["h"], state["w"], state["labels"], state["dloss"],
                                               frozen=c["frozen"])
        return dict(loss=loss, lse=lse, dh=dh) if c["frozen"] else dict(loss=loss, lse=lse, dh=dh, dw=dw)
    if kind.startswith("norm"):
        train = kind == "norm_train"
        y, s, stats = ops.norm_forward(state["x"], state["gain"], state["shift"], rms=c["rms"], eps=EPS,
                                       res=state["res"], with_stats=train)
        out = dict(y=y)
        if state["res"] is not None:
            out["s"] = s
        if train:
            out["dgain"] = torch.zeros(c["d"], device=DEV)
            if state["shift"] is not None:
                out["dshift"] = torch.zeros(c["d"], device=DEV)
            out["dx"] = ops.norm_backward(state["dy"], s, state["gain"], stats, rms=c["rms"], dskip=state["dskip"],
                                          dgain=out["dgain"], dshift=out.get("dshift"))
        return out
    how = dict(positions=state["positions"], freq=state["freq"], sections=_sections(c))
    q, k = ops.rotary(state["q"], state["k"], **how)
    out = dict(q_turned=q, k_turned=k)
    if kind == "rotary_train":
        out["dq_turned"], out["dk_turned"] = ops.rotary(state["dq"], state["dk"], inverse=True, **how)
    return out


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("ce_train", "ce_score", "next"):
        n, d, vocab = max(1, round(case["n"] * case["counted"])), case["d"], case["vocab"]
        if kind != "ce_train":
            return {"bytes": es * d * (n + vocab) + 8 * case["n"], "flops": 2 * n * d * vocab}
        tensors, products = (1, 2) if case["frozen"] else (2, 3)
        return {"bytes": es * d * (n + case["n"] + tensors * vocab) + 16 * case["n"],
                "flops": 2 * products * n * d * vocab}
    if kind in ("norm", "norm_train"):
        tensors = 4 if case["res"] else 2
        if kind == "norm_train":  # s (or x) again, dy, dskip, dx; the same rows would have to stay on the chip otherwise
            tensors += 4 if case["res"] else 3
        return {"bytes": es * tensors * case["rows"] * case["d"], "flops": 0}
    one = case["batch"] * case["rows"] * (case["heads"] + case["kv_heads"]) * case["dh"]
    return {"bytes": es * one * (4 if kind == "rotary_train" else 2), "flops": 0}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "next":
        x = st["h"].double() @ st["w"].double().T
        best, token = torch.log_softmax(x, 1).max(1)
        return {"token": token.int(), "logprob": best}
    if kind.startswith("ce"):
        return _exact_ce(case, st)
    if kind.startswith("norm"):
        return _exact_norm(case, st)
    out = {"q_turned": _exact_turn(case, st, st["q"], 1), "k_turned": _exact_turn(case, st, st["k"], 1)}
    if kind == "rotary_train":
        out["dq_turned"], out["dk_turned"] = _exact_turn(case, st, st["dq"], -1), _exact_turn(case, st, st["dk"], -1)
    return out


def _exact_ce(case, st):
    n, d, vocab = case["n"], case["d"], case["vocab"]
    f64 = dict(dtype=torch.float64, device=DEV)
    out = {"loss": torch.zeros(n, **f64), "lse": torch.zeros(n, **f64)}
    train = case["kind"] == "ce_train"
    if train:
        out["dh"] = torch.zeros(n, d, **f64)
        if not case["frozen"]:
            out["dw"] = torch.zeros(vocab, d, **f64)
    w = st["w"].double()
    for at in range(0, n, 1024):
        rows = slice(at, min(n, at + 1024))
        counts = (st["labels"][rows] >= 0).double()
        label = st["labels"][rows].long().clamp(min=0)
        h = st["h"][rows].double()
        logp = torch.log_softmax(h @ w.T, 1)
        mine = logp[torch.arange(len(label), device=DEV), label]
        out["loss"][rows] = -mine * counts
        out["lse"][rows] = (torch.linalg.vecdot(h, w[label]) - mine) * counts
        if train:
            logp.exp_()
            logp[torch.arange(len(label), device=DEV), label] = torch.expm1(mine)
            logp *= (counts * st["dloss"][rows].double())[:, None]
            out["dh"][rows] = logp @ w
            if not case["frozen"]:
                out["dw"].addmm_(logp.T, h)
    return out


def _exact_norm(case, st):
    s = st["x"]
    if case["res"]:  # what is stored is what is normalised
        s = (s.double() + st["res"].double()).to(s.dtype)
    x, gain, d = s.double(), st["gain"].double(), case["d"]
    mean = torch.zeros_like(x[:, 0]) if case["rms"] else x.sum(1) / d
    away = x - mean[:, None]
    deviation = torch.sqrt(torch.linalg.vecdot(away, away) / d + EPS)
    unit = away / deviation[:, None]
    out = {"y": unit * gain + (st["shift"].double() if case["shift"] else 0.0)}
    if case["res"]:
        out["s"] = x
    if case["kind"] == "norm_train":
        dy = st["dy"].double()
        dunit = dy * gain
        along = torch.linalg.vecdot(dunit, unit) / d
        dx = dunit - along[:, None] * unit
        if not case["rms"]:
            dx -= (dunit.sum(1) / d)[:, None]
        dx /= deviation[:, None]
        if case["res"]:
            dx += st["dskip"].double()
        out["dx"], out["dgain"] = dx, torch.einsum("nd,nd->d", dy, unit)
        if case["shift"]:
            out["dshift"] = dy.sum(0)
    return out


def _exact_turn(case, st, x, sign):
    pairs = sum(_sections(case))
    which = [a for a, m in enumerate(_sections(case)) for _ in range(m)]
    z = torch.complex(x[..., :pairs].double(), x[..., pairs:2 * pairs].double())
    turn = torch.stack([st["positions"][a].double() * f for a, f in zip(which, _frequencies(case))], -1)
    z = z * torch.polar(torch.ones_like(turn), sign * turn)[:, :, None]
    return torch.cat((z.real, z.imag, x[..., 2 * pairs:].double()), -1)
