"""What the vocabulary head and its gradients leave of quantities that the formulas let cancel, and what they make of
infinities and of batches in pieces, against float64.  head_reference.py has the roundings' sizes."""
import math

import pytest

import head_reference as R

pytestmark = pytest.mark.gpu


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape, std=1.0, dtype=torch.float32: (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def near_classes(n, d, V, apart, ahead, seed=0):
    """bf16 classes that have most of their rows in common, and labels whose logits lead the others' mean by `ahead`."""
    import torch
    r = gen(n + 3 * d + V + seed)
    w = (r(1, d, std=d ** -0.5) + apart * r(V, d, std=d ** -0.5)).bfloat16()
    labels = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n + seed)).cuda()
    lead = w[labels].float() - w.float().mean(0)
    h = (r(n, d) + lead * (ahead / lead.square().sum(1, keepdim=True))).bfloat16()
    return h, w, labels.int(), r(n, std=1.0 / n)


def dh_apart(h, w, labels, dloss, counted):
    """(dh, bound): an entry of P that is off by e moves dh by e (w - w[label]), as the entries of a row sum to zero.  Of what all
    classes have in common only the fp32 sums' roundings are left: of the products (8 sqrt(V) e), of the row of P (64 entries to a
    thread, a tree of 8, runs of 16384 columns) and of the two roundings that put w[label] in."""
    import torch
    V, d = w.shape
    u = R.half_step(torch.bfloat16)
    up = u * u if counted <= 64 else u
    H, W, lab = h.double(), w.double(), labels.long()[:, None]
    s, A = H @ W.T, H.abs() @ W.abs().T
    lse = torch.logsumexp(s, 1, keepdim=True)
    logp = s - lse
    p = logp.exp()
    g = dloss.double()[:, None]
    P = g * p.scatter(1, lab, torch.expm1(logp.gather(1, lab)))
    es = 8 * math.sqrt(d) * R.E * A
    elog = es + (p * es).sum(1, keepdim=True) + 4 * R.E * (1 + logp.abs())
    # a logit waits in fp16 below its tile's maximum, which is at most lse: half a step of that distance
    eP = g.abs() * p * (elog + 2.0 ** -11 * logp.abs() + 2.0 ** -24)
    eP = (eP + up * (P.abs() + eP) * 1.01).scatter(1, lab, 0.0)
    dh, size, apart = P @ W, P.abs() @ W.abs(), torch.empty_like(H)
    for i in range(len(h)):
        apart[i] = eP[i] @ (W - W[lab[i, 0]]).abs()
    own = W[lab[:, 0]].abs() * P.abs().sum(1, keepdim=True)
    e = apart + 8 * math.sqrt(V) * R.E * size + (64 + 8 + V / 16384 + 4) * R.E * own + 4 * R.E * size
    return dh, 1.01 * e + u * (dh.abs() + e) * 1.01


@pytest.mark.parametrize("ahead", [0.0, 3.0, 9.0, 20.0])
@pytest.mark.parametrize("n,d,V,apart", [
    (1, 64, 40, 0.1), (64, 64, 40, 0.03), (65, 64, 40, 0.1), (65, 64, 40, 0.03), (1000, 64, 40, 0.03),  # dh without shares
    (64, 128, 3000, 0.03), (65, 128, 3000, 0.03), (300, 72, 1100, 0.1), (70, 24, 40000, 0.03), (20, 24, 40000, 0.1),  # in shares; runs of columns
    (4100, 2304, 520, 0.03)])  # 256 rows and columns to a tile
def test_dh_of_classes_that_differ_little(n, d, V, apart, ahead):
    import torch
    from paper_2502_19864_amd import operators as ops
    h, w, labels, dloss = near_classes(n, d, V, apart, ahead)
    loss, lse, dh, dw = ops.vocab_ce_train(h, w, labels, dloss)
    some = torch.arange(n, device="cuda")[:: max(1, n // 64)]
    want, bound = dh_apart(h[some], w, labels[some], dloss[some], n)
    R.check("dh", dh[some], want, bound)
    # the same rows among others that do not count, and in a batch of another size
    wide = torch.full((2 * n + 3, d), math.nan, dtype=h.dtype, device="cuda")
    lab, g = torch.full((2 * n + 3,), -1, dtype=torch.int32, device="cuda"), torch.zeros(2 * n + 3, device="cuda")
    wide[3::2], lab[3::2], g[3::2] = h, labels, dloss
    among = ops.vocab_ce_train(wide, w, lab, g, frozen=True)[2]
    assert not among[:3].any() and not among[4::2].any()
    R.check("dh", among[3::2][some], want, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [30.0, 300.0, 3000.0])
@pytest.mark.parametrize("n,d,V", [(5, 40, 96), (70, 40, 96), (300, 136, 200)])
def test_what_all_logits_share_reaches_no_gradient(n, d, V, offset, dtype):
    """One column of w is 1 and one of h large: every logit has it, and the entries of a row of P sum to zero however
    large it is, so that column of dh vanishes."""
    import torch
    from paper_2502_19864_amd import operators as ops
    t, r = torch.bfloat16 if dtype == "bf16" else torch.float32, gen(n + V)
    h, w = r(n, d, dtype=t), r(V, d, std=2 * d ** -0.5, dtype=t)
    h[:, d - 1], w[:, d - 1] = offset, 1.0
    labels = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n)).cuda()
    dloss = r(n)
    dh = ops.vocab_ce_train(h, w, labels.int(), dloss)[2][:, d - 1]
    logp = torch.log_softmax(h.double() @ w.double().T, 1)
    p, mine = logp.exp(), logp.gather(1, labels[:, None])
    # the entries: an argument's roundings and the function's two steps, whatever the logits' own; then a sum of V products, and
    # in bf16 the row's sum and the product that take it off
    entries = (p * 4 * R.E * (3 + logp.abs())).sum(1) + 8 * R.E * (1 - mine[:, 0])
    sums = (8 * math.sqrt(V) + 80) * R.E * 2
    R.check("dh", dh, torch.zeros(n, dtype=torch.float64, device="cuda"), dloss.double().abs() * (entries + sums))


@pytest.mark.parametrize("dtype,n,d,V", [
    ("bf16", 3, 1000, 40000), ("bf16", 20, 2056, 40000), ("bf16", 3, 72, 700), ("bf16", 20, 264, 700), ("bf16", 9, 512, 3000),  # few rows
    ("bf16", 70, 200, 900), ("bf16", 100, 8, 900), ("bf16", 190, 200, 60000), ("bf16", 512, 136, 30000), ("bf16", 128, 128, 500),  # tiles of 128, 192, 256 rows
    ("f32", 5, 33, 300), ("f32", 70, 2, 90), ("f32", 70, 133, 16400), ("f32", 1500, 6, 1502), ("f32", 100, 64, 16400)])
def test_infinite_weights(dtype, n, d, V):
    """An infinity in w makes the logits of its class infinite or, against the other sign of h, leaves it out; it reaches no
    other class, whatever of its row a kernel reads past d."""
    import torch
    from paper_2502_19864_amd import operators as ops
    t, r = torch.bfloat16 if dtype == "bf16" else torch.float32, gen(n + d + V)
    h, w = r(n, d, dtype=t), r(V, d, std=d ** -0.5, dtype=t)
    labels = torch.randint(0, V - 8, (n,), generator=torch.Generator().manual_seed(n)).cuda().int()
    for at in sorted({0, d // 2, d - 8 if d > 8 else d - 1, d - 1}):
        h[:, at] = -1.0
        for k, v in enumerate((V - 1, V - 7)):
            out, far = w.clone(), w.clone()
            out[v, at], far[v, at] = math.inf, 2.0 ** 100
            loss, lse = ops.vocab_ce_forward(h, out, labels)
            want = ops.vocab_ce_forward(h, far, labels)  # exp of -2^100 is 0 too
            assert torch.equal(loss, want[0]) and torch.equal(lse, want[1]) and torch.isfinite(loss).all()
            assert all(torch.equal(a, b) for a, b in zip(ops.vocab_next(h, out), ops.vocab_next(h, far)))
            if k == 0:
                dloss = torch.full((n,), 1.0 / n, device="cuda")
                got, want = ops.vocab_ce_train(h, out, labels, dloss), ops.vocab_ce_train(h, far, labels, dloss)
                rest = torch.arange(d, device="cuda") != at
                assert all(torch.equal(a, b) for a, b in zip(got[:2], want[:2]))
                assert torch.equal(got[2][:, rest], want[2][:, rest]) and torch.equal(got[3], want[3])
            out[v, at] = -math.inf  # against h's -1: the largest logit there is
            token, logprob = ops.vocab_next(h, out)
            assert (token == v).all() and torch.isnan(logprob).all()
            assert torch.isnan(ops.vocab_ce_forward(h, out, labels)[0]).all()


PIECES = [  # dtype, d, vocab, rows that are held at a time, rows that count in the next piece
    ("bf16", 8, 300007, 3328, 0), ("bf16", 8, 300007, 3328, 1), ("bf16", 8, 300007, 3328, 64), ("bf16", 8, 300007, 3328, 65),
    ("bf16", 264, 300007, 3328, 200), ("bf16", 8, 4096, 262144, 37001), ("bf16", 136, 4096, 262144, 63),  # 256-wide dw; dw in shares
    ("f32", 8, 300007, 1536, 1), ("f32", 264, 300007, 1536, 200), ("f32", 72, 4096, 131072, 8900)]  # 128-wide tiles, dw in shares


@pytest.mark.parametrize("dtype,d,V,held,after", PIECES)
def test_pieces_of_rows(dtype, d, V, held, after):
    """More logits than are held at a time, `after` rows that count in the second piece: dw is carried from piece to piece, and few
    rows there are in two parts."""
    import torch
    from paper_2502_19864_amd import binding as B
    from paper_2502_19864_amd import operators as ops
    t, code, es = (torch.bfloat16, B.BF16, 2) if dtype == "bf16" else (torch.float32, B.F32, 4)
    counted, n = held + after, held + 260 + after
    assert held == (1 << 31) // es // ((V + 63) // 64 * 64) // 256 * 256 < n <= 2 * held  # two pieces
    plan = lambda rows: B.ringada_vocab_plan(B.VocabDesc(code, rows, d, V))[1]
    if dtype == "bf16":
        assert plan(n) - plan(held) >= 4 * V * d  # dw between them
    h, w, labels, dloss = near_classes(n, d, V, 0.3, 3.0)
    h, w = h.to(t), w.to(t)
    off = torch.randperm(n, generator=torch.Generator().manual_seed(d))[:n - counted].cuda()
    labels[off], h[off] = -1, math.nan
    loss, lse, dh, dw = ops.vocab_ce_train(h, w, labels, dloss)
    assert not any(x[off].any() for x in (loss, lse, dh))
    at = (labels >= 0).nonzero()[:, 0]
    step = 16384 if V < 10000 else 1024
    want_dw = bound_dw = 0.0
    for piece in (at[:held], at[held:])[:1 + (after > 0)]:
        for rows in piece.split(step):
            assert len(rows) > 64 or len(piece) <= 64  # two parts where the piece has them
            want = R.vocab(h[rows], w, labels[rows], dloss[rows])
            for name, got in (("loss", loss), ("lse", lse), ("dh", dh)):
                R.check(name, got[rows], *want[name])
            # the sums of these rows, each within its bound, are added in fp32: a few dozen additions in a row at most, of which
            # the bound of a sum of m products, 8 sqrt(m) e, has its share
            want_dw = want_dw + want["dw"][0]
            bound_dw = bound_dw + want["dw"][1] * (1 + 8 / math.sqrt(len(rows)))
    R.check("dw", dw, want_dw, bound_dw)
    if dtype == "bf16":
        for rows, m in ((at[:held:held // 5], held), (at[held::13], after)):
            if len(rows):
                R.check("dh", dh[rows], *dh_apart(h[rows], w, labels[rows], dloss[rows], m))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decoding_keeps_to_the_whole_sequence(dtype):
    """Token by token against a cache and the whole sequence at once, within what their roundings leave; a step whose newest
    key is missing is told apart by that.

    Seven tensors lie between the embedding and the logits (norm, projection, rotary, attention, projection, sum, norm), so
    two paths differ by up to 14 independent roundings, each of 0.0017 (bf16; fp32: 8 half steps, as a product's sum has more
    of them) of an element in the mean square.  A logit takes them by its terms' root of squares; six times that is not
    reached in some 10^5 logits."""
    import torch
    from test_gpu_head_operators import block_and_head, dt

    from paper_2502_19864_amd import operators as ops
    B, S, d, H, Hkv, dh, V = 3, 24, 128, 4, 2, 64, 900
    p, ids = block_and_head(dtype, B, S, d, H, Hkv, dh, V, 5)
    ids = ids.clamp(min=0)[:, :S]
    w = gen(7)(V, d, std=0.5, dtype=dt(dtype))  # not the embedding, under which every input is its own next token, surely
    freq = ops.rotary_frequencies((dh // 2,), device="cuda")
    cache = torch.zeros(2, B, S, Hkv, dh, dtype=dt(dtype), device="cuda")
    pos = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S).contiguous()
    each = 0.0017 if dtype == "bf16" else 8 * R.E

    def project(x, at, **out):
        n, _, _ = ops.norm_forward(x, p["g1"], rms=True, with_stats=False)
        qkv = (n.reshape(-1, d) @ p["wqkv"]).view(B, -1, H + 2 * Hkv, dh)
        q, k = ops.rotary(qkv[:, :, :H], qkv[:, :, H:H + Hkv], positions=at, freq=freq, **out)
        return q, k, qkv[:, :, H + Hkv:]

    def finish(x, o):
        a = (o.reshape(-1, H * dh) @ p["wo"]).view(x.shape)
        return ops.norm_forward(a, p["g2"], rms=True, res=x, with_stats=False)[0]
    q, k, v = project(p["emb"][ids], pos)
    whole = finish(p["emb"][ids], ops.attention_forward(q, k, v, causal=True)[0])
    token, logprob = ops.vocab_next(whole, w)
    sure, off = 0, 0
    for t in range(S):
        x = p["emb"][ids[:, t:t + 1]]
        q, _, v = project(x, pos[:, t:t + 1].contiguous(), out_k=cache[0][:, t:t + 1])
        cache[1][:, t:t + 1] = v

        def step(keys):
            lens = torch.full((B,), keys, dtype=torch.int32, device="cuda")
            return ops.vocab_next(finish(x, ops.attention_forward(q, cache[0], cache[1], causal=True, len_k=lens)[0])[:, 0], w)
        terms = whole[:, t].double().square() @ w.double().square().T
        tol = 6 * math.sqrt(14) * each * terms.amax(1).sqrt()
        tok, lp = step(t + 1)
        assert ((lp - logprob[:, t]).abs() <= tol).all()
        best = (whole[:, t].double() @ w.double().T).topk(2, 1).values
        clear = best[:, 0] - best[:, 1] > 2 * tol
        assert torch.equal(tok[clear], token[:, t][clear])
        sure += int(clear.sum())
        if t:
            tok, lp = step(t)
            off += int(((lp - logprob[:, t]).abs() > tol).sum())
    assert sure >= B * S // 2
    assert off >= B * S // 4
