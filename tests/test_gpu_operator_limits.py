"""The block operators at the ends of their documented ranges."""
import math

import pytest

import philox_vectors as P

pytestmark = pytest.mark.gpu


def signed(x):
    return x - 2 ** 64 if x >= 2 ** 63 else x


def keeps(x, at, want, rng, site):
    """Elements at .. at + 7 of x stay exactly while the threshold is at most their 16 bits `want`."""
    from paper_2502_19864_amd import operators as ops
    for h in want:
        for thr in (h, h + 1):
            if thr > 65535:
                continue
            x[at:at + 8] = 1
            ops.dropout(x, thr / 65536, rng, site, out=x)
            assert (x[at:at + 8] != 0).tolist() == [w >= thr for w in want], (at, thr)


@pytest.mark.parametrize("i,n", [(0, 8), (2, 8 * 0x243f6a88 + 8), (1, 1 << 35)])
def test_dropout_gives_the_published_vectors(i, n):
    """The generator's vectors read back from the mask of the elements that have their counter; the last one is
    the last element of the largest tensor (64 GiB)."""
    import torch

    if torch.cuda.mem_get_info()[0] < 2 * n + (8 << 30):
        pytest.skip("not enough free memory")
    counter, key, out = P.VECTORS[i]
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    rng = torch.tensor([signed(key[0] | key[1] << 32), signed(counter[2] | counter[3] << 32)], device="cuda")
    keeps(x, 8 * counter[0], [h for w in out for h in (w & 0xFFFF, w >> 16)], rng, counter[1])
    if n > 1 << 34:  # both sides of where the launch takes a second row of workgroups
        for at in ((1 << 34) - 8, 1 << 34):
            want = P.halves(at // 8, key[0] | key[1] << 32, counter[2] | counter[3] << 32, counter[1])
            keeps(x, at, want, rng, counter[1])
    del x
    torch.cuda.empty_cache()


def T(dtype, H, Hkv, dh, Sq, Sk, **kw):
    from test_gpu_operators import A
    return A(dtype, 1, H, Hkv, dh, Sq, Sk, **kw)


@pytest.mark.parametrize("c", [
    T("f32", 8, 1, 64, 512, 512, causal=True),
    T("f32", 16, 2, 16, 305, 305, window=100),
    T("f32", 16, 1, 40, 400, 400, causal=True, window=80, sinks=3, nb=16, dist=20),
    T("bf16", 32, 1, 128, 600, 600, causal=True),
    T("bf16", 8, 1, 64, 2048, 128),
    T("bf16", 4, 4, 64, 700, 700, causal=True),
], ids=str)
def test_few_key_blocks_met_by_many_query_tiles(c):
    """The dK/dV pass of few key blocks, or of blocks that every query sees, dealt to many workgroups."""
    import operator_reference as R
    from test_gpu_operators import make, run
    t = make(c)
    got = run(t)
    want = R.attention(t["q"], t["k"], t["v"], t["do"], lowp=c["dtype"] == "bf16", d_exact=bool(c["nb"]), **t["how"])
    for n in got:
        R.check(n, got[n], *want[n])


@pytest.mark.parametrize("B,Sq,Sk,H", [(1, 1, 700, 4), (1, 90, 90, 1), (3, 1, 1, 2), (1, 1, 1, 1)])
def test_any_stride_of_a_single_entry(B, Sq, Sk, H):
    """Dimensions of one entry have the strides that torch happens to give them."""
    import torch

    from paper_2502_19864_amd import operators as ops

    def odd(x):
        return x.as_strided(x.shape, [s if n > 1 else 13 + (1 << 30) for n, s in zip(x.shape[:3], x.stride())] + [1])

    g = torch.Generator().manual_seed(2)
    q, do, k, v = (torch.randn(B, S, H, 64, generator=g).bfloat16().cuda() for S in (Sq, Sq, Sk, Sk))
    o, lse = ops.attention_forward(q, k, v, causal=True)
    grads = ops.attention_backward(do, q, k, v, o, lse, causal=True)
    outs = [odd(torch.empty_like(x)) for x in (q, q, k, v)]
    o2, lse2 = ops.attention_forward(odd(q), odd(k), odd(v), causal=True, out=outs[0])
    ops.attention_backward(odd(do), odd(q), odd(k), odd(v), o2, lse2, causal=True, dq=outs[1], dk=outs[2], dv=outs[3])
    for a, b in zip((o, lse) + grads, (o2, lse2) + tuple(outs[1:])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("c", [T("bf16", 8, 2, 128, 1, 3000, causal=True), T("f32", 4, 2, 40, 3, 2000, causal=True, nb=8, dist=20),
                               T("bf16", 4, 2, 64, 100, 100), T("f32", 2, 2, 100, 60, 60, causal=True),
                               T("bf16", 64, 32, 64, 300, 300, causal=True, window=90, sinks=3),
                               T("bf16", 32, 32, 128, 270, 270, causal=True, nb=16, dist=30)], ids=str)
def test_a_nan_among_the_visible_keys_is_not_lost(c):
    """Rows that see a key of NaN are NaN, in lse too, whichever kernels they take; the others are as they were."""
    import torch
    from paper_2502_19864_amd import operators as ops
    from test_gpu_operators import make

    t = make(c)
    o, lse = ops.attention_forward(t["q"], t["k"], t["v"], **t["how"])
    k = t["k"].clone()
    k[:, c["Sk"] - 1] = float("nan")
    o2, lse2 = ops.attention_forward(t["q"], k, t["v"], **t["how"])
    hit = torch.ones(c["Sq"], dtype=torch.bool, device="cuda")
    if c["causal"]:  # the last key is its own query's alone
        hit[:-1] = False
    assert torch.isnan(o2[:, hit]).all() and torch.isnan(lse2[:, :, hit]).all()
    assert torch.equal(o2[:, ~hit], o[:, ~hit]) and torch.equal(lse2[:, :, ~hit], lse[:, :, ~hit])


@pytest.mark.parametrize("dtype,dh,H,Hkv,S,nb,window", [
    ("bf16", 64, 2, 2, 100, 0, 0), ("bf16", 128, 2, 2, 100, 16, 0), ("f32", 40, 2, 2, 100, 16, 0), ("f32", 100, 2, 2, 60, 0, 0),
    ("bf16", 64, 4, 2, 200, 0, 70), ("bf16", 128, 4, 2, 200, 16, 70), ("f32", 40, 4, 2, 200, 16, 0), ("f32", 100, 4, 1, 100, 0, 0),
    ("bf16", 64, 32, 8, 900, 16, 70), ("bf16", 128, 32, 8, 900, 0, 70), ("bf16", 128, 32, 8, 900, 16, 0), ("f32", 40, 32, 8, 900, 0, 70)])
def test_zeros_stay_zeros_beside_infinities(dtype, dh, H, Hkv, S, nb, window):
    """Infinities and NaN within one sequence: its rows past the lengths and those that see nothing are zeros as
    ever, and the other sequence is as it was."""
    import torch
    from test_gpu_operators import A, make, run

    lq, lk = S - 9, S - 21  # the first twelve rows stand before the first key
    c = A(dtype, 2, H, Hkv, dh, S, causal=True, window=window, sinks=2 if window else 0, nb=nb, dist=20 if nb else 0,
          len_q=[lq, S], len_k=[lk, S])
    t = make(c, layout="cache")
    clean = run(t)
    inf = float("inf")
    t["v"][0, 3] = inf
    t["v"][0, lk - 1, :, 1:] = float("nan")
    t["k"][0, 7, :, 0] = -inf
    t["do"][0, 20] = inf
    t["do"][0, lq - 1, :, :1] = float("nan")
    got = run(t)
    for n in ("o", "dq"):
        assert torch.equal(got[n][1], clean[n][1]), n
        assert (got[n][0, :12] == 0).all() and (got[n][0, lq:] == 0).all(), n
    for n in ("dk", "dv"):
        assert torch.equal(got[n][1], clean[n][1]), n
        assert (got[n][0, lk:] == 0).all(), n
    assert (got["lse"][0, :, :12] == -inf).all() and (got["lse"][0, :, lq:] == -inf).all()
    assert torch.equal(got["lse"][1], clean["lse"][1])


FAR = [("bf16", 64, 2, 2, 100, 100), ("bf16", 128, 2, 2, 90, 90), ("f32", 40, 2, 2, 100, 100), ("f32", 100, 2, 2, 60, 60),
       ("bf16", 64, 4, 2, 150, 200), ("bf16", 128, 4, 2, 200, 200), ("f32", 40, 4, 2, 200, 200), ("f32", 100, 4, 1, 100, 130),
       ("bf16", 64, 64, 16, 300, 300), ("bf16", 128, 64, 64, 270, 270), ("f32", 40, 64, 16, 270, 270), ("f32", 100, 64, 32, 270, 270),
       ("bf16", 128, 8, 2, 3, 1500)]


@pytest.mark.parametrize("big", [-1e9, -1e6, 1000.0])
@pytest.mark.parametrize("frozen", [False, True])
@pytest.mark.parametrize("dtype,dh,H,Hkv,Sq,Sk", FAR)
def test_entries_of_large_magnitude_in_all_that_a_row_sees(dtype, dh, H, Hkv, Sq, Sk, frozen, big):
    """A table of one value throughout is no bias: where the scores are all the same (q or k is zero), so that fp32
    holds their sums with it exactly, outputs and gradients are those of a table of zeros, as head 0's is."""
    import operator_reference as R
    import torch
    from test_gpu_operators import A, make, run

    c = A(dtype, 2, H, Hkv, dh, Sq, Sk, causal=True, nb=8, dist=20, len_q=[Sq, Sq - Sq // 3], len_k=[Sk, Sk - Sk // 4])
    t = make(c, layout="cache")
    plain = torch.zeros_like(t["table"])
    t["table"].fill_(big)
    t["table"][:, 0] = 0
    for zero in ("q", "k"):
        z = dict(t)
        z[zero] = torch.zeros_like(t[zero])
        got = run(z, frozen)
        want = R.attention(z["q"], z["k"], z["v"], z["do"], lowp=dtype == "bf16", d_exact=not frozen, **dict(t["how"], table=plain))
        shift = t["table"][0].double().cpu() / math.log(2)
        for n in got:
            if n == "lse":
                at = ~torch.isinf(want[n][0])
                w = torch.where(at, want[n][0] + shift[None, :, None], want[n][0])
                R.check(n, got[n], w, want[n][1] + 2.0 ** -22 * w.abs().nan_to_num(posinf=0))
            else:
                R.check(n + " " + zero, got[n], *want[n])


def test_a_captured_stage_keeps_its_memory():
    """A graph of a stage with options goes on working after a larger batch, other options and another
    generator have replaced what it uses, and writes into nobody else's memory."""
    import torch
    from paper_2502_19864_amd import operators as ops
    from paper_2502_19864_amd.stage import Stage
    from paper_2502_19864_amd.workloads import Workload, make_inputs

    w = Workload("captured", "bert", "bf16", 2, 256, 4, 512, 64, 150, 2, 0, "dy", 3120)
    inp = make_inputs(w)
    st = Stage(w, inp, max_batch=8)
    try:
        def table(seed):
            g = torch.Generator().manual_seed(seed)
            return torch.randn(16, 4, generator=g).to(st.dev)

        bucket = ops.relpos_buckets(16, 30, True, st.dev)
        gt = torch.zeros(16, 4, device=st.dev)
        st.set_attention(60, 1, table(1), bucket, gt)
        st.set_dropout(0.1, torch.tensor([5, 6], dtype=torch.int64, device=st.dev), 4)
        x, dy = st.upload(inp["x"]), st.upload(inp["dy"])
        y, dx = st.empty(*x.shape), st.empty(*x.shape)

        def step():
            gt.zero_()
            st.zero_grads()
            st.forward(x, y, -1)
            st.backward(dy, -1, dx)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, gt)]
        sizes = [t.numel() for t in (st.stash, st.scratch, st.attention[4])]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        big, out = st.empty(8, w.seq, w.d_model).normal_(), st.empty(8, w.seq, w.d_model)
        st.set_attention(30, 2, table(2), bucket.clone(), torch.zeros_like(gt))
        st.set_dropout(0.2, torch.tensor([7, 8], dtype=torch.int64, device=st.dev), 0)
        st.forward(big, out, -1)
        st.backward(big, -1, torch.empty_like(big))
        torch.cuda.synchronize()
        junk = [torch.full((n,), 91, dtype=torch.uint8, device=st.dev) for n in sizes + [16, 128, 256] * 8]
        for _ in range(3):
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip((y, dx, gt), want):
                assert torch.equal(a, b)
            assert all(bool((j == 91).all()) for j in junk)
    finally:
        st.close()


@pytest.mark.parametrize("table", ["none", "frozen", "trained"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 40), ("f32", 100)])
def test_rows_that_fill_the_gpu_over_several_tiles(dtype, dh, causal, table):
    """Every form of the passes whose waves take a block of rows each: masks, window, sinks, lengths, shared heads
    and a bias whose reach ends inside the sequence; 1.6 times the blocks from which these forms are taken."""
    import operator_reference as R
    from test_gpu_operators import A, make, run

    c = A(dtype, 2, 24, 6, dh, 520, causal=causal, window=150, sinks=5, nb=0 if table == "none" else 16, dist=0 if
          table == "none" else 40, len_q=[520, 333], len_k=[520, 333])
    t = make(c)
    got = run(t, frozen_table=table == "frozen")
    want = R.attention(t["q"], t["k"], t["v"], t["do"], lowp=dtype == "bf16", d_exact=table == "trained", **t["how"])
    assert ("dtable" in got) == (table == "trained")
    for n in got:
        print(n, R.check(n, got[n], *want[n]), flush=True)
