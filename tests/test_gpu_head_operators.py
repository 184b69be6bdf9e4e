"""Norms, the rotary embedding and the vocabulary head on the GPU against float64, alone and
together.  head_reference.py has the references and the bounds."""
import math

import pytest

import head_reference as R

pytestmark = pytest.mark.gpu


def dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape, std=1.0, mean=0.0, dtype=torch.float32: (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


# ---------------------------------------------------------------- norms
NORMS = [  # dtype, rows, d: pieces of a row, threads per row, and both sides of each division
    ("bf16", 1, 1), ("bf16", 3, 7), ("bf16", 1, 4096), ("bf16", 5, 511), ("bf16", 130, 512), ("bf16", 67, 520),
    ("bf16", 4, 1024), ("bf16", 3000, 768), ("bf16", 33, 1029), ("bf16", 9, 2048), ("bf16", 700, 2056), ("bf16", 6, 8192),
    ("bf16", 3, 8200), ("bf16", 2, 16384), ("bf16", 5, 16383), ("f32", 1, 2), ("f32", 129, 128), ("f32", 77, 255),
    ("f32", 4, 1025), ("f32", 600, 1028), ("f32", 3, 4096), ("f32", 7, 4099), ("f32", 2, 16384), ("bf16", 5000, 64),
    ("f32", 9, 400), ("f32", 5, 401), ("f32", 30, 800), ("f32", 6, 801), ("f32", 5, 3001), ("f32", 4, 8000), ("f32", 2, 16383),
    ("bf16", 11, 1001), ("bf16", 3, 5001),
]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("dtype,rows,d", NORMS)
def test_norm(dtype, rows, d, res, rms):
    import torch
    from paper_2502_19864_amd import operators as ops
    t, r = dt(dtype), gen(rows * 31 + d)
    x = r(rows, d, std=2.0, mean=0.5, dtype=t)
    add = r(rows, d, dtype=t) if res else None
    gain, shift = r(d, std=0.3, mean=1.0, dtype=t), None if rms else r(d, dtype=t)
    y, s, stats = ops.norm_forward(x, gain, shift, rms=rms, eps=1e-5, res=add)
    if res:
        exact = x.double() + add.double()
        # rounded in fp32 first, which moves a tie at most
        R.check("s", s, exact, R.half_step(t) * exact.abs() * (1 + 2.0 ** -14))
    else:
        assert s is x
    dy, skip = r(rows, d, std=0.1, dtype=t), r(rows, d, std=0.1, dtype=t) if res else None
    dgain, dshift = r(d), r(d)
    g0, b0 = dgain.clone(), dshift.clone()
    dx = ops.norm_backward(dy, s, gain, stats, rms=rms, dskip=skip, dgain=dgain, dshift=dshift)
    want = R.norm(s, gain, shift, rms, 1e-5, dy, skip)
    R.check("y", y, *want["y"])
    R.check("dx", dx, *want["dx"])
    for name, got, base in (("dgain", dgain, g0), ("dshift", dshift, b0)):
        v, e = want[name]
        R.check(name, got, v + base.double(), e + R.E * (v + base.double()).abs() + 1e-30)
    # without the parameters' gradients, and one of them alone
    assert torch.equal(ops.norm_backward(dy, s, gain, stats, rms=rms, dskip=skip), dx)
    only = torch.zeros_like(dgain)
    ops.norm_backward(dy, s, gain, stats, rms=rms, dskip=skip, dshift=only)
    R.check("dshift", only, *want["dshift"])
    assert torch.equal(ops.norm_forward(x, gain, shift, rms=rms, eps=1e-5, res=add, with_stats=False)[0], y)


def test_norm_against_differences():
    """dx, dgain and dshift in fp32 against central differences of the float64 formula."""
    import torch
    from paper_2502_19864_amd import operators as ops
    r = gen(3)
    for rms in (False, True):
        x, gain, shift, dy = r(4, 24), r(24, mean=1.0), r(24), r(4, 24)
        y, s, stats = ops.norm_forward(x, gain, shift, rms=rms)
        dgain, dshift = torch.zeros(24, device="cuda"), torch.zeros(24, device="cuda")
        dx = ops.norm_backward(dy, s, gain, stats, rms=rms, dgain=dgain, dshift=dshift)

        def f(a, g, b):
            c = a if rms else a - a.mean(1, keepdim=True)
            return ((c * (c.square().mean(1, keepdim=True) + 1e-5).rsqrt() * g + b) * dy.double()).sum()
        args = [x.double(), gain.double(), shift.double()]
        for i, got in enumerate((dx, dgain, dshift)):
            flat = args[i].reshape(-1)
            for j in range(0, flat.numel(), 5):
                keep, step = flat[j].item(), 1e-5
                flat[j] = keep + step
                hi = f(*args)
                flat[j] = keep - step
                lo = f(*args)
                flat[j] = keep
                # differences: third derivatives of order 10 times step^2, and 1e-16 / step of the sum; the kernel: 1e-5
                assert abs((hi - lo).item() / (2 * step) - got.reshape(-1)[j].item()) <= 2e-5 * (1 + abs(got.reshape(-1)[j].item()))


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 300), ("f32", 100), ("bf16", 4096)])
def test_norm_strides_and_places(dtype, d):
    """Rows of wider tensors, broadcast rows, misaligned rows; results over inputs; bits that repeat."""
    import torch
    from paper_2502_19864_amd import operators as ops
    t, r = dt(dtype), gen(d)
    rows = 21
    wide = r(rows, 2 * d + 3, dtype=t)
    for x in (wide[:, :d], wide[:, 1:d + 1], wide[:1, 2:d + 2].expand(rows, d), wide[:, d:2 * d]):
        gain = r(d + 1, mean=1.0, dtype=t)[1:]
        res, dy = r(rows, d, dtype=t), r(rows, d, dtype=t)
        plain = ops.norm_forward(x.contiguous(), gain.clone(), res=res)
        out = torch.full((rows, d + 5), 7.0, dtype=t, device="cuda")
        got = ops.norm_forward(x, gain, res=res, out=out[:, 3:d + 3])
        for a, b in zip(got, plain):
            R.check("strided", a, b.double(), 64 * R.E * 8 * (1 + b.double().abs()) + 2 * R.half_step(t) * b.double().abs())
        assert (out[:, :3] == 7).all() and (out[:, d + 3:] == 7).all()
        over = res.clone()
        y, s, stats = ops.norm_forward(x, gain, res=over, out=over, out_sum=torch.empty_like(over))
        assert torch.equal(y, got[0]) and y is over
        keep = dy.clone()
        g1, g2 = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        dx = ops.norm_backward(dy, s, gain, stats, dskip=res, dgain=g1)
        assert torch.equal(ops.norm_backward(keep, s, gain, stats, dskip=res, dgain=g2, out=keep), dx)
        assert torch.equal(g1, g2)
        assert torch.equal(ops.norm_backward(dy, s, gain, stats, dskip=res, out=s), dx)


def test_norm_rows_stay_apart():
    """A row of infinities or NaN reaches no other row."""
    import torch
    from paper_2502_19864_amd import operators as ops
    r = gen(9)
    for d in (64, 1024, 4096):
        x, gain = r(9, d, dtype=torch.bfloat16), r(d, mean=1.0, dtype=torch.bfloat16)
        clean = ops.norm_forward(x, gain)[0]
        bad = x.clone()
        bad[4] = math.nan
        bad[7, 5] = math.inf
        y, s, stats = ops.norm_forward(bad, gain)
        dx = ops.norm_backward(x, s, gain, stats)
        for i in range(9):
            if i in (4, 7):
                assert torch.isnan(y[i]).any()
            else:
                assert torch.equal(y[i], clean[i]) and torch.isfinite(dx[i]).all()


# ---------------------------------------------------------------- rotary
ROTARY = [  # dtype, B, S, H, Hkv, dh, sections, first position
    ("bf16", 1, 1, 1, 0, 64, (32,), 0), ("bf16", 3, 1, 32, 8, 128, (64,), 100003), ("bf16", 2, 37, 4, 2, 64, (32,), 0),
    ("bf16", 2, 300, 4, 1, 128, (16, 24, 24), 1 << 20), ("bf16", 1, 70, 3, 3, 80, (20, 20), 5),
    ("bf16", 2, 33, 2, 2, 96, (12,), -40), ("bf16", 1, 9, 2, 1, 256, (8, 8, 8, 8), 2 ** 31 - 600), ("bf16", 1, 2100, 2, 1, 64, (16,), 0),
    ("f32", 1, 5, 1, 1, 2, (1,), 0), ("f32", 2, 65, 3, 1, 40, (5, 15), 1 << 20), ("f32", 3, 500, 2, 2, 6, (1, 1, 1), 77),
    ("f32", 1, 7, 2, 0, 1024, (512,), 10 ** 6), ("f32", 1, 1200, 2, 1, 128, (64,), 0), ("bf16", 2, 3, 5, 2, 1024, (200, 300), 9),
    ("f32", 1, 3, 2, 1, 17, (4,), 0),
]


def positions(sections, b, s, first, seed):
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    p = torch.stack([first + torch.randint(0, 600 if first < 2 ** 30 else 599, (b, s), generator=g) for _ in sections])
    return p.int().cuda()


@pytest.mark.parametrize("dtype,B,S,H,Hkv,dh,sections,first", ROTARY)
def test_rotary(dtype, B, S, H, Hkv, dh, sections, first):
    import torch
    from paper_2502_19864_amd import operators as ops
    t, r = dt(dtype), gen(B * S + dh)
    qkv = r(B, S, H + 2 * max(1, Hkv), dh, dtype=t) if dtype == "f32" or dh % 8 == 0 else None
    q, k = qkv[:, :, :H], qkv[:, :, H:H + Hkv] if Hkv else None
    freq = ops.rotary_frequencies(sections, shared=len(sections) == 2, device="cuda")
    pos = positions(sections, B, S, first, dh)
    for inverse in (False, True):
        how = dict(positions=pos, freq=freq, sections=sections, inverse=inverse)
        a, b = ops.rotary(q, k, **how)
        R.check("q", a, *R.rotary(q, pos, freq, sections, inverse))
        if Hkv:
            R.check("k", b, *R.rotary(k, pos, freq, sections, inverse))
        else:
            assert b is None
        # in place, and head by head in memory
        q2 = q.clone()
        assert torch.equal(ops.rotary(q2, None, out_q=q2, **how)[0], a)
        heads = torch.empty(B, H, S, dh, dtype=t, device="cuda").transpose(1, 2)
        ops.rotary(q, None, out_q=heads, **how)
        assert torch.equal(heads, a)


def test_rotary_is_the_stages_rope():
    """One axis: pairs (i, i + dh / 2) by position theta^(-2 i / dh), as the pre-RMS stages rotate."""
    import torch
    from paper_2502_19864_amd import operators as ops
    x = gen(1)(1, 50, 2, 64)
    freq = ops.rotary_frequencies((32,), 10000.0, device="cuda")
    got, _ = ops.rotary(x, positions=torch.arange(50, dtype=torch.int32, device="cuda")[None], freq=freq)
    i = torch.arange(32, device="cuda", dtype=torch.float64)
    a = torch.arange(50, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-2 * i / 64)
    c, s = a.cos()[None, :, None], a.sin()[None, :, None]
    lo, hi = x[..., :32].double(), x[..., 32:].double()
    want = torch.cat((lo * c - hi * s, hi * c + lo * s), -1)
    R.check("rope", got, want, 10 * R.E * (lo.abs() + hi.abs()).repeat(1, 1, 1, 2) + R.E * want.abs())


# ---------------------------------------------------------------- vocabulary head
VOCAB = [  # dtype, rows, d, vocab, share of rows that count
    ("f32", 1, 1, 1, 1.0), ("f32", 3, 5, 2, 1.0), ("f32", 128, 128, 512, 1.0), ("f32", 37, 130, 129, 0.6), ("f32", 300, 65, 1000, 0.5),
    ("f32", 17, 1027, 333, 1.0), ("f32", 1, 77, 5003, 1.0),
    ("bf16", 1, 8, 1, 1.0), ("bf16", 1, 64, 65, 1.0), ("bf16", 2, 24, 127, 1.0), ("bf16", 16, 512, 4099, 1.0), ("bf16", 17, 264, 2000, 0.9),
    ("bf16", 64, 128, 3000, 1.0), ("bf16", 65, 768, 1283, 0.7), ("bf16", 127, 136, 1024, 1.0), ("bf16", 128, 64, 128, 1.0),
    ("bf16", 129, 320, 640, 1.0), ("bf16", 257, 768, 5001, 0.15), ("bf16", 500, 1024, 777, 0.9), ("bf16", 1000, 256, 9001, 1.0),
    ("bf16", 20000, 16, 130, 0.5), ("bf16", 16385, 24, 70, 0.2), ("f32", 17408, 5, 40, 0.3), ("bf16", 12000, 200, 86, 1.0), ("f32", 9000, 40, 50, 0.9),
    ("bf16", 700, 2056, 1030, 1.0), ("bf16", 300, 2304, 3000, 1.0), ("bf16", 190, 640, 4000, 0.9), ("f32", 600, 260, 3001, 1.0), ("f32", 700, 257, 2001, 0.8),
    ("f32", 1500, 1030, 1100, 1.0), ("f32", 400, 1500, 1200, 0.3), ("bf16", 33, 512, 3001, 1.0), ("bf16", 3, 16384, 300, 1.0), ("bf16", 4, 16376, 200, 1.0),
    ("bf16", 32, 4096, 5000, 1.0), ("bf16", 32, 64, 20000, 0.7), ("bf16", 9, 1000, 100000, 1.0), ("bf16", 4500, 4096, 1000, 1.0),
    ("f32", 2100, 1000, 300, 1.0), ("f32", 1500, 1032, 1400, 1.0), ("f32", 1200, 1100, 2000, 1.0), ("bf16", 16, 2048, 17000, 1.0),
    ("bf16", 20, 2048, 17000, 0.9), ("bf16", 20, 512, 33000, 1.0), ("bf16", 20, 2048, 3000, 1.0), ("bf16", 1000, 72, 16000, 1.0), ("bf16", 2, 4096, 40000, 1.0), ("bf16", 1500, 520, 300, 0.8), ("bf16", 40, 16, 70000, 1.0),
    ("f32", 1500, 1, 1600, 1.0), ("f32", 1500, 3, 1601, 0.9), ("f32", 1500, 4, 1602, 1.0), ("f32", 1501, 6, 1603, 1.0), ("f32", 17000, 3, 41, 1.0), ("f32", 17000, 7, 42, 0.8),
    ("f32", 1400, 2051, 1411, 1.0), ("f32", 1300, 1022, 1999, 0.7), ("f32", 10, 1157, 2562, 1.0),
    ("bf16", 4, 8, 196, 0.3), ("bf16", 63, 72, 1100, 1.0), ("bf16", 4500, 4096, 1000, 0.01), ("bf16", 200, 2048, 4200, 0.2), ("bf16", 64, 2056, 3001, 1.0),
]


def head(dtype, n, d, V, counted, seed=0, std=1.0):
    import torch
    t, r = dt(dtype), gen(n * 7 + d * 3 + V + seed)
    w = r(V, d, std=std * d ** -0.5, dtype=t)
    g = torch.Generator()
    g.manual_seed(n + V + seed)
    labels = torch.randint(0, V, (n,), generator=g)
    h = (r(n, d) + torch.rand(n, 1, generator=g).cuda() * 10 * w[labels.cuda()].float()).to(t)
    off = torch.rand(n, generator=g) >= counted
    labels[off] = torch.tensor([-1, V, -100, 2 ** 31 - 1])[torch.arange(int(off.sum())) % 4]
    return h, w, labels.int().cuda(), r(n, std=1.0 / n)


@pytest.mark.parametrize("dtype,n,d,V,counted", VOCAB)
def test_vocab(dtype, n, d, V, counted):
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = head(dtype, n, d, V, counted)
    want = R.vocab(h, w, labels, dloss)
    loss, lse, dh, dw = ops.vocab_ce_train(h, w, labels, dloss)
    for name, got in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
        R.check(name, got, *want[name])
    f = ops.vocab_ce_forward(h, w, labels)
    for name, got in zip(("loss", "lse"), f):
        R.check(name, got, *want[name])
    off = (labels < 0) | (labels >= V)
    for t in (loss, lse, dh, *f):
        assert not t[off].any()
    frozen = ops.vocab_ce_train(h, w, labels, dloss, frozen=True)
    assert frozen[3] is None and torch.equal(frozen[2], dh) and torch.equal(frozen[0], loss)
    again = ops.vocab_ce_train(h, w, labels, dloss)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, lse, dh, dw)))


@pytest.mark.parametrize("dtype,n,d,V,counted", VOCAB)
def test_vocab_next(dtype, n, d, V, counted):
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, _, _ = head(dtype, n, d, V, 1.0)
    token, logprob = ops.vocab_next(h, w)
    s = h.double() @ w.double().T
    A = h.double().abs() @ w.double().abs().T
    best, err = s.amax(1), (8 * math.sqrt(d) * R.E * A).amax(1)
    mine = s.gather(1, token.long()[:, None])[:, 0]
    assert token.dtype is torch.int32 and (best - mine <= 2 * err).all()
    sure = (s >= (best - 2 * err)[:, None]).sum(1) == 1
    assert torch.equal(token[sure].long(), s.argmax(1)[sure])
    want = R.vocab(h, w, token)["loss"]
    R.check("logprob", logprob, -want[0], want[1])


@pytest.mark.parametrize("n", [1, 5, 40, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocab_next_takes_the_lowest_of_equals(dtype, n):
    """Rows of w that repeat: the first of them, wherever the copies lie."""
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, _, _ = head(dtype, n, 64, 3000, 1.0, seed=4)
    token, logprob = ops.vocab_next(h, w)
    for copies in ([1, 2], [700, 64], [2999, 1500]):
        w2 = torch.cat((w[:copies[0]], w, w[copies[1]:]))  # every row but some stands twice
        first = [(w2 == w[j]).all(1).nonzero()[0, 0] for j in token.tolist()]
        assert torch.equal(ops.vocab_next(h, w2)[0].long(), torch.stack(first))
    zero = ops.vocab_next(torch.zeros_like(h), w)
    assert (zero[0] == 0).all()
    R.check("logprob", zero[1], torch.full((n,), -math.log(3000), device="cuda", dtype=torch.float64), torch.full((n,), 64 * R.E * 8, device="cuda", dtype=torch.float64))


@pytest.mark.parametrize("n,d,V", [(1, 8, 60), (3, 8, 200), (20, 16, 700), (64, 32, 1500), (64, 24, 40000)])
def test_few_rows_keep_what_is_left_of_dh(n, d, V):
    """Classes that differ little: dh is what their differences leave, and P's roundings must not reach it."""
    import torch
    from paper_2502_19864_amd import operators as ops
    for seed in range(6):
        h, w, labels, dloss = head("bf16", n, d, V, 1.0, seed=seed)
        w = (w[:1] + 0.05 * w).contiguous()
        want = R.vocab(h, w, labels, dloss)
        for name, got in zip(("loss", "lse", "dh", "dw"), ops.vocab_ce_train(h, w, labels, dloss)):
            R.check(name, got, *want[name])


@pytest.mark.parametrize("n,d,V", [(1500, 133, 1502), (1500, 4, 1501), (40, 133, 300), (17000, 130, 40)])
def test_f32_vocab_rows_from_any_address(n, d, V):
    """Four floats at a time or not, the same products in the same order."""
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = head("f32", n, d, V, 0.9, seed=d)
    want = ops.vocab_ce_train(h, w, labels, dloss)
    for pad in (1, 2, 7):
        wide = [torch.full((x.shape[0], d + pad + 1), math.nan, device="cuda") for x in (h, w)]
        hs, ws = (x[:, pad:pad + d].copy_(y) for x, y in zip(wide, (h, w)))
        assert all(torch.equal(a, b) for a, b in zip(ops.vocab_ce_train(hs, ws, labels, dloss), want))
        assert all(torch.equal(a, b) for a, b in zip(ops.vocab_next(hs, ws), ops.vocab_next(h, w)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_do_not_count_reach_nothing(dtype):
    """NaN and infinities in their h and dloss; a batch where none counts."""
    import torch
    from paper_2502_19864_amd import operators as ops
    for n in (5, 70, 300):
        h, w, labels, dloss = head(dtype, n, 72, 600, 0.5, seed=n)
        off = (labels < 0) | (labels >= 600)
        assert off.any() and not off.all()
        clean = ops.vocab_ce_train(h, w, labels, dloss)
        h[off], dloss[off] = math.nan, math.inf
        h[off.nonzero()[0, 0]] = -math.inf
        got = ops.vocab_ce_train(h, w, labels, dloss)
        assert all(torch.equal(a, b) for a, b in zip(got, clean))
        assert all(torch.equal(a, b) for a, b in zip(ops.vocab_ce_forward(h, w, labels), ops.vocab_ce_forward(torch.where(off[:, None], 0, h), w, labels)))
        none = ops.vocab_ce_train(h, w, torch.full_like(labels, -1), dloss, dh=torch.full_like(h, 3), dw=torch.full_like(w, 3))
        assert not any(t.any() for t in none)


def test_vocab_sure_rows_and_large_logits():
    """Losses near zero keep their digits; logits of some hundreds overflow nothing."""
    import torch
    from paper_2502_19864_amd import operators as ops
    for dtype in ("bf16", "f32"):
        for n in (7, 150):
            h, w, labels, dloss = head(dtype, n, 256, 500, 1.0, seed=1)
            h = (2.0 * w[labels.long()].float() * torch.arange(1, n + 1, device="cuda")[:, None] * (400 / n)).to(h.dtype)
            want = R.vocab(h, w, labels, dloss)
            got = ops.vocab_ce_train(h, w, labels, dloss)
            for name, g in zip(("loss", "lse", "dh", "dw"), got):
                R.check(name, g, *want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocab_strides(dtype):
    """h, w and the gradients as columns of wider tensors, h with leading dimensions."""
    import torch
    from paper_2502_19864_amd import operators as ops
    for n, d, V in ((6, 64, 300), (150, 136, 400)):
        h, w, labels, dloss = head(dtype, n, d, V, 0.8)
        base = ops.vocab_ce_train(h, w, labels, dloss)
        wide = lambda t: torch.full((t.shape[0], t.shape[1] + 24), 5.0, dtype=t.dtype, device="cuda")
        H, W, DH, DW = wide(h), wide(w), wide(h), wide(w)
        cut = lambda t: t[:, 8:t.shape[1] - 16]
        cut(H).copy_(h)
        cut(W).copy_(w)
        got = ops.vocab_ce_train(cut(H), cut(W), labels, dloss, dh=cut(DH), dw=cut(DW))
        assert all(torch.equal(a, b) for a, b in zip(got, base))
        for t in (DH, DW):
            assert (t[:, :8] == 5).all() and (t[:, -16:] == 5).all()
        assert all(torch.equal(a, b) for a, b in zip(ops.vocab_next(cut(H), cut(W)), ops.vocab_next(h, w)))
        lead = ops.vocab_ce_train(h.view(2, n // 2, d), w, labels.view(2, -1), dloss.view(2, -1))
        assert lead[0].shape == (2, n // 2) and lead[2].shape == (2, n // 2, d)
        assert all(torch.equal(a.reshape(b.shape), b) for a, b in zip(lead, base))


@pytest.mark.parametrize("dtype,n,V", [("bf16", 5, 1100), ("bf16", 40, 1100), ("bf16", 300, 1100), ("f32", 20, 700), ("f32", 3000, 700)])
def test_vocab_rows_far_apart(dtype, n, V):
    """The largest row strides: w and dw span more than 2^32 bytes, their tiles almost as much."""
    import torch
    from paper_2502_19864_amd import operators as ops
    d, ld = 264, 1 << 22
    h, w, labels, dloss = head(dtype, n, d, V, 0.9)
    far = lambda rows: torch.empty((rows - 1) * ld + d, dtype=h.dtype, device="cuda").as_strided((rows, d), (ld, 1))
    w2, dw2 = far(V).copy_(w), far(V)
    got, want = ops.vocab_ce_train(h, w2, labels, dloss, dw=dw2), ops.vocab_ce_train(h, w, labels, dloss)
    assert got[3] is dw2 and all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(ops.vocab_ce_forward(h, w2, labels), ops.vocab_ce_forward(h, w, labels)))
    assert all(torch.equal(a, b) for a, b in zip(ops.vocab_next(h, w2), ops.vocab_next(h, w)))
    if n <= 300:
        h2, dh2 = far(n).copy_(h), far(n)
        got = ops.vocab_ce_train(h2, w, labels, dloss, dh=dh2)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,n,d,V,counted", [c for c in VOCAB if c[1] * c[3] < 1 << 25][::2] + [("bf16", 700, 72, 900, 0.05), ("bf16", 90, 72, 900, 0.0)])
def test_vocab_workspace_may_hold_anything(dtype, n, d, V, counted):
    import torch
    from paper_2502_19864_amd import binding as B
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = head(dtype, n, d, V, counted)
    want, scored, nexts = ops.vocab_ce_train(h, w, labels, dloss), ops.vocab_ce_forward(h, w, labels), ops.vocab_next(h, w)
    desc = B.VocabDesc(B.BF16 if dtype == "bf16" else B.F32, n, d, V)
    sizes, stream = B.ringada_vocab_plan(desc), torch.cuda.current_stream().cuda_stream
    hr, wr = B.Rows(h.data_ptr(), d), B.Rows(w.data_ptr(), d)
    for fill in (255, 127):
        loss, lse, dh, dw = (torch.full_like(t, 3) for t in want)
        ws = torch.full((sizes[1],), fill, dtype=torch.uint8, device="cuda")
        t = B.VocabTensors(hr, wr, labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), dloss.data_ptr(), B.Rows(dh.data_ptr(), d),
                           B.Rows(dw.data_ptr(), d))
        B.ringada_vocab_ce(stream, desc, t, ws, sizes[1])
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, dh, dw), want))
        loss, lse = (torch.full_like(t, 3) for t in scored)
        ws = torch.full((sizes[0],), fill, dtype=torch.uint8, device="cuda")
        t = B.VocabTensors(hr, wr, labels.data_ptr(), loss.data_ptr(), lse.data_ptr(), None, B.Rows(0, 0), B.Rows(0, 0))
        B.ringada_vocab_ce(stream, desc, t, ws, sizes[0])
        assert all(torch.equal(a, b) for a, b in zip((loss, lse), scored))
        token, logprob = (torch.full_like(t, 3) for t in nexts)
        ws = torch.full((sizes[2],), fill, dtype=torch.uint8, device="cuda")
        B.ringada_vocab_next(stream, desc, hr, wr, token, logprob, ws, sizes[2])
        assert torch.equal(token, nexts[0]) and torch.equal(logprob, nexts[1])


def test_vocab_gradients_one_at_a_time():
    """dw without dh, through the C names; of rows with one dloss, several, and none in the first."""
    import torch
    from paper_2502_19864_amd import binding as B
    from paper_2502_19864_amd import operators as ops
    for dtype, code in (("bf16", B.BF16), ("f32", B.F32)):
        n, d, V = 300, 72, 500
        h, w, labels, dloss = head(dtype, n, d, V, 0.7)
        first = int(((labels >= 0) & (labels < V)).nonzero()[0])
        for k in range(4):
            g = [dloss, torch.full_like(dloss, -3e-5), dloss * 1e4, dloss.clone()][k]
            if k == 3:
                g[first] = 0
            want = R.vocab(h, w, labels, g)
            loss, lse, dh, dw = ops.vocab_ce_train(h, w, labels, g)
            R.check("dh", dh, *want["dh"])
            R.check("dw", dw, *want["dw"])
            alone = torch.full_like(w, 7)
            size = B.ringada_vocab_plan(B.VocabDesc(code, n, d, V))[1]
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
            t = B.VocabTensors(B.Rows(h.data_ptr(), d), B.Rows(w.data_ptr(), d), labels.data_ptr(), loss.data_ptr(), lse.data_ptr(),
                               g.data_ptr(), B.Rows(0, 0), B.Rows(alone.data_ptr(), d))
            B.ringada_vocab_ce(torch.cuda.current_stream().cuda_stream, B.VocabDesc(code, n, d, V), t, ws, size)
            assert torch.equal(alone, dw)


def test_vocab_infinities_and_nan_that_count():
    """A row that counts and holds a NaN or an infinity is NaN, and so is dw; the other rows are as without it."""
    import torch
    from paper_2502_19864_amd import operators as ops
    for dtype in ("bf16", "f32"):
        for n in (6, 140):
            h, w, labels, dloss = head(dtype, n, 64, 700, 1.0)
            clean = ops.vocab_ce_train(h, w, labels, dloss)
            bad = h.clone()
            bad[3, 5], bad[n - 1, 0] = math.nan, math.inf
            loss, lse, dh, dw = ops.vocab_ce_train(bad, w, labels, dloss)
            sane = torch.ones(n, dtype=torch.bool, device="cuda")
            sane[3] = sane[n - 1] = False
            for got, want in ((loss, clean[0]), (lse, clean[1]), (dh, clean[2])):
                assert torch.equal(got[sane], want[sane]) and torch.isnan(got[~sane]).all()
            assert torch.isnan(dw).all()
            f = ops.vocab_ce_forward(bad, w, labels)
            assert all(torch.isnan(x[~sane]).all() and torch.isfinite(x[sane]).all() for x in f)
            token, logprob = ops.vocab_next(bad, w)
            assert ((token >= 0) & (token < 700)).all() and torch.isnan(logprob[~sane]).all()
            assert torch.equal(token[sane], ops.vocab_next(h, w)[0][sane])


def test_vocab_against_differences():
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = head("f32", 9, 12, 31, 0.7)
    dloss = gen(5)(9)
    _, _, dh, dw = ops.vocab_ce_train(h, w, labels, dloss)
    keep = (labels >= 0) & (labels < 31)

    def f(a, b):
        logp = torch.log_softmax(a[keep] @ b.T, 1)
        return -(logp.gather(1, labels[keep].long()[:, None])[:, 0] * dloss[keep].double()).sum()
    args = [h.double(), w.double()]
    for i, got in enumerate((dh, dw)):
        flat = args[i].reshape(-1)
        for j in range(0, flat.numel(), 7):
            at, step = flat[j].item(), 1e-5
            flat[j] = at + step
            hi = f(*args)
            flat[j] = at - step
            lo = f(*args)
            flat[j] = at
            # step^2 times third derivatives (of order 10), 1e-15 / step; the kernel's 1e-6
            assert abs((hi - lo).item() / (2 * step) - got.reshape(-1)[j].item()) <= 1e-5


@pytest.mark.parametrize("dtype,n,V", [("bf16", 3700, 300007), ("bf16", 3390, 300007), ("f32", 1900, 300007)])
def test_vocab_in_pieces(dtype, n, V):
    """More logits than are held at a time: pieces of the rows, dw summed over them; the rows that count end
    inside the first, or are all in it."""
    import torch
    from paper_2502_19864_amd import binding as B
    from paper_2502_19864_amd import operators as ops
    desc = B.VocabDesc(B.BF16 if dtype == "bf16" else B.F32, n, 8, V)
    assert B.ringada_vocab_plan(desc)[1] < 4 * (1 << 30)
    for counted in (1.0, 0.9, 0.3):
        h, w, labels, dloss = head(dtype, n, 8, V, counted)
        want = R.vocab(h, w, labels, dloss)
        for name, g in zip(("loss", "lse", "dh", "dw"), ops.vocab_ce_train(h, w, labels, dloss)):
            R.check(name, g, *want[name])


def test_vocab_long_sums_are_cut():
    """dh over 300007 classes, with tiles enough for every CU."""
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = head("bf16", 3300, 2304, 300007, 1.0)
    loss, lse, dh, _ = ops.vocab_ce_train(h, w, labels, dloss, frozen=True)
    rows = slice(1000, 1200)
    want = R.vocab(h[rows], w, labels[rows], dloss[rows])
    for name, got in (("loss", loss), ("lse", lse), ("dh", dh)):
        R.check(name, got[rows], *want[name])


# ---------------------------------------------------------------- streams and graphs
def calls(seed, n=70):
    """One call of each operator as a function of no arguments that returns its outputs."""
    import torch
    from paper_2502_19864_amd import operators as ops
    r = gen(seed)
    b = torch.bfloat16
    x, res, gain, dy = r(n, 768, dtype=b), r(n, 768, dtype=b), r(768, mean=1.0, dtype=b), r(n, 768, dtype=b)
    q, pos = r(2, n, 4, 64, dtype=b), positions((32,), 2, n, 5, seed)
    freq = ops.rotary_frequencies((32,), device="cuda")
    h, w, labels, dloss = head("bf16", n, 256, 3001, 0.7, seed)

    def norm():
        y, s, stats = ops.norm_forward(x, gain, res=res)
        dgain = torch.zeros(768, device="cuda")
        return y, s, ops.norm_backward(dy, s, gain, stats, dskip=res, dgain=dgain), dgain
    return [norm, lambda: ops.rotary(q, q, positions=pos, freq=freq), lambda: ops.vocab_ce_train(h, w, labels, dloss),
            lambda: ops.vocab_ce_forward(h[:9], w, labels[:9]), lambda: ops.vocab_next(h[:3], w)]


@pytest.mark.parametrize("i", range(5))
def test_captured_calls(i):
    """Two graphs with workspaces of their own, replayed in turn with eager work between, give the eager results."""
    import torch
    fs = [calls(1)[i], calls(2)[i]]
    eager = [f() for f in fs]
    graphs, outs = [], []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for f in fs:
            f()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(f())
            graphs.append(g)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, out, want in zip(graphs, outs, eager):
            for t in out:
                t.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            assert all(torch.equal(a, b) for a, b in zip(fs[0](), eager[0]))


def test_streams_at_once():
    import torch
    fs = [f for seed in (1, 2) for f in calls(seed, 200)]
    want = [f() for f in fs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in fs]
    got = [[] for _ in fs]
    for _ in range(4):
        for i, (f, s) in enumerate(zip(fs, streams)):
            with torch.cuda.stream(s):
                got[i].append(f())
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for outs in g:
            assert all(torch.equal(a, b) for a, b in zip(outs, w))


# ---------------------------------------------------------------- together
def block_and_head(dtype, B, S, d, H, Hkv, dh, V, seed):
    import torch
    r, t = gen(seed), dt(dtype)
    g = torch.Generator()
    g.manual_seed(seed)
    ids = torch.randint(0, V, (B, S + 1), generator=g).cuda()
    ids[1, S // 2:] = -1  # a shorter sequence
    p = dict(emb=r(V, d, std=0.5, dtype=t), g1=r(d, mean=1.0, std=0.1, dtype=t), g2=r(d, mean=1.0, std=0.1, dtype=t),
             wqkv=r(d, (H + 2 * Hkv) * dh, std=d ** -0.5, dtype=t), wo=r(H * dh, d, std=(H * dh) ** -0.5, dtype=t))
    return p, ids


def library_step(p, ids, H, Hkv, dh, freq, lens):
    """A pre-norm attention block and a tied head from the library's calls: losses, gradients."""
    import torch
    from paper_2502_19864_amd import operators as ops
    B, S = ids.shape[0], ids.shape[1] - 1
    d = p["emb"].shape[1]
    labels = ids[:, 1:].int().contiguous()
    pos = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S).contiguous()
    x = p["emb"][ids[:, :-1].clamp(min=0)]
    n1, s1, st1 = ops.norm_forward(x, p["g1"], rms=True)
    qkv = (n1.view(-1, d) @ p["wqkv"]).view(B, S, H + 2 * Hkv, dh)
    v = qkv[:, :, H + Hkv:]
    q, k = ops.rotary(qkv[:, :, :H], qkv[:, :, H:H + Hkv], positions=pos, freq=freq)
    how = dict(causal=True, len_q=lens, len_k=lens)
    o, lse = ops.attention_forward(q, k, v, **how)
    a = (o.reshape(-1, H * dh) @ p["wo"]).view(B, S, d)
    n2, s2, st2 = ops.norm_forward(a, p["g2"], rms=True, res=x)
    count = (labels >= 0).sum()
    dloss = (labels >= 0).float() / count
    loss, _, dn2, dw = ops.vocab_ce_train(n2, p["emb"], labels, dloss)
    g = {"w": dw, "g1": torch.zeros(d, device="cuda"), "g2": torch.zeros(d, device="cuda")}
    ds2 = ops.norm_backward(dn2, s2, p["g2"], st2, rms=True, dgain=g["g2"])
    da = ds2.view(-1, d)
    do = (da @ p["wo"].t()).view(B, S, H, dh)
    g["wo"] = o.reshape(-1, H * dh).t() @ da
    dqkv = torch.empty_like(qkv)
    dq, dk, _ = ops.attention_backward(do, q, k, v, o, lse, dv=dqkv[:, :, H + Hkv:], **how)
    ops.rotary(dq, dk, positions=pos, freq=freq, inverse=True, out_q=dqkv[:, :, :H], out_k=dqkv[:, :, H:H + Hkv])
    g["wqkv"] = n1.view(-1, d).t() @ dqkv.view(B * S, -1)
    dn1 = (dqkv.view(B * S, -1) @ p["wqkv"].t()).view(B, S, d)
    g["x"] = ops.norm_backward(dn1, s1, p["g1"], st1, rms=True, dskip=ds2, dgain=g["g1"])
    return loss.sum() / count, g


def reference_step(p, ids, H, Hkv, dh, freq):
    """The same in float64 with torch's autograd, sequence by sequence."""
    import torch
    P = {n: t.double().requires_grad_() for n, t in p.items()}
    x = p["emb"].double()[ids[:, :-1].clamp(min=0)].requires_grad_()
    w = P["emb"]
    rms = lambda z, g: z * (z.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * g
    total, count = 0.0, (ids[:, 1:] >= 0).sum()
    for b in range(ids.shape[0]):
        n = int((ids[b, :-1] >= 0).sum())
        z = x[b, :n]
        qkv = (rms(z, P["g1"]) @ P["wqkv"]).view(n, H + 2 * Hkv, dh)
        angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * freq
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        turn = lambda y: torch.cat((y[..., :dh // 2] * c - y[..., dh // 2:] * s, y[..., dh // 2:] * c + y[..., :dh // 2] * s), -1)
        q, k, v = turn(qkv[:, :H]), turn(qkv[:, H:H + Hkv]), qkv[:, H + Hkv:]
        out = []
        for h in range(H):
            sc = q[:, h] @ k[:, h * Hkv // H].T * dh ** -0.5
            sc = sc.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
            out.append(torch.softmax(sc, 1) @ v[:, h * Hkv // H])
        s2 = z + torch.cat(out, 1) @ P["wo"]
        logits = rms(s2, P["g2"]) @ w.T
        lab = ids[b, 1:n + 1].long()
        has = lab >= 0
        total = total - torch.log_softmax(logits, 1)[has].gather(1, lab[has][:, None]).sum() / count
    total.backward()
    return total.detach(), {"w": w.grad, "g1": P["g1"].grad, "g2": P["g2"].grad, "wo": P["wo"].grad, "wqkv": P["wqkv"].grad, "x": x.grad}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_from_the_calls(dtype):
    import torch
    from paper_2502_19864_amd import operators as ops
    B, S, d, H, Hkv, dh, V = 2, 50, 128, 4, 2, 64, 700
    p, ids = block_and_head(dtype, B, S, d, H, Hkv, dh, V, 3)
    freq = ops.rotary_frequencies((dh // 2,), device="cuda")
    lens = (ids[:, :-1] >= 0).sum(1).int()
    loss, g = library_step(p, ids, H, Hkv, dh, freq, lens)
    want, gw = reference_step(p, ids, H, Hkv, dh, freq)
    # a dozen roundings between the input and the furthest gradient, each of half a step of the values' size, add up as
    # their squares and are amplified at most some times by the norms: 12 half steps of the largest value
    u = R.half_step(dt(dtype))
    assert abs(loss.item() - want.item()) <= 12 * u * abs(want.item())
    for n, t in g.items():
        off = (t.double() - gw[n]).norm() / gw[n].norm()
        assert off <= 12 * max(u, 8 * R.E), (n, off.item())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decoding_from_the_calls(dtype):
    """Token by token against a cache: the same tokens and log-probabilities as the whole sequence at once."""
    import torch
    from paper_2502_19864_amd import operators as ops
    B, S, d, H, Hkv, dh, V = 3, 24, 128, 4, 2, 64, 900
    p, ids = block_and_head(dtype, B, S, d, H, Hkv, dh, V, 5)
    ids = ids.clamp(min=0)[:, :S]
    freq = ops.rotary_frequencies((dh // 2,), device="cuda")
    cache = torch.zeros(2, B, S, Hkv, dh, dtype=dt(dtype), device="cuda")

    def project(x):
        n, _, _ = ops.norm_forward(x, p["g1"], rms=True, with_stats=False)
        return (n.reshape(-1, d) @ p["wqkv"]).view(B, -1, H + 2 * Hkv, dh)

    def finish(x, o):
        a = (o.reshape(-1, H * dh) @ p["wo"]).view(x.shape)
        return ops.norm_forward(a, p["g2"], rms=True, res=x, with_stats=False)[0]
    x = p["emb"][ids]
    qkv = project(x)
    pos = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S).contiguous()
    q, k = ops.rotary(qkv[:, :, :H], qkv[:, :, H:H + Hkv], positions=pos, freq=freq)
    whole = finish(x, ops.attention_forward(q, k, qkv[:, :, H + Hkv:], causal=True)[0])
    token, logprob = ops.vocab_next(whole, p["emb"])
    for t in range(S):
        x1 = p["emb"][ids[:, t:t + 1]]
        one = project(x1)
        q1, _ = ops.rotary(one[:, :, :H], one[:, :, H:H + Hkv], positions=pos[:, t:t + 1].contiguous(), freq=freq,
                           out_k=cache[0][:, t:t + 1])
        cache[1][:, t:t + 1] = one[:, :, H + Hkv:]
        lens = torch.full((B,), t + 1, dtype=torch.int32, device="cuda")
        y = finish(x1, ops.attention_forward(q1, cache[0], cache[1], causal=True, len_k=lens)[0])
        tok, lp = ops.vocab_next(y[:, 0], p["emb"])
        # a dozen roundings of logits of some units; tokens agree where the runner-up is further away than that
        u = 12 * R.half_step(dt(dtype)) * 8 + 1e-5
        assert (lp - logprob[:, t]).abs().max() <= u * 4
        logits = whole[:, t].double() @ p["emb"].double().T
        top = logits.topk(2, 1).values
        sure = top[:, 0] - top[:, 1] > u * 4
        assert torch.equal(tok[sure], token[:, t][sure])
