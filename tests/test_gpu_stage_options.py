"""Stages with a windowed attention, a learned relative position bias and dropout, against the
oracle: outputs, input and adapter gradients, the table's gradient; options on and off
again; the schedule driver with dropout."""
import numpy as np
import pytest

import oracle as O
from gpu_run import run_gpu
from helpers import Checker, oracle_desc, to64
from paper_2502_19864_amd import binding as B
from paper_2502_19864_amd.stage import Stage
from paper_2502_19864_amd.workloads import Workload, make_inputs
from stage_options import keep, score_add, table_grad

pytestmark = pytest.mark.gpu

CASES = {
    # name: (workload, window, sinks, buckets, R, dropout)
    "f32": (Workload("opt_f32", "bert", "f32", 2, 128, 2, 512, 16, 32, 4, 0, "dy", 3101), 7, 1, 16, 12, 0.2),
    "f32_single": (Workload("opt_f32s", "bert", "f32", 2, 96, 3, 128, 16, 21, 3, 0, "dy", 3102, placement="ffn"),
                   0, 0, 8, 9, 0.4),
    "bert_128": (Workload("opt_b128", "bert", "bf16", 2, 256, 4, 512, 64, 128, 2, 0, "dy", 3103), 0, 0, 32, 100, 0.1),
    "bert_window": (Workload("opt_bw", "bert", "bf16", 2, 256, 4, 512, 64, 203, 2, 0, "dy", 3104), 40, 2, 0, 0, 0.0),
    "bert_single": (Workload("opt_bs", "bert", "bf16", 2, 256, 4, 512, 64, 150, 2, 0, "dy", 3105, placement="ffn"),
                    60, 1, 16, 30, 0.1),
    "bert_dh128": (Workload("opt_bd", "bert", "bf16", 2, 512, 4, 512, 64, 150, 2, 0, "dy", 3106), 50, 3, 0, 0, 0.1),
    "llama": (Workload("opt_l", "llama", "bf16", 2, 256, 2, 512, 64, 300, 2, 0, "dy", 3107), 65, 4, 32, 128, 0.1),
    "llama_64": (Workload("opt_l64", "llama", "bf16", 2, 256, 4, 512, 64, 140, 2, 0, "dy", 3108), 30, 0, 0, 0, 0.1),
    # rotated heads of short sequences, and of rows that fill the GPU
    "llama_short": (Workload("opt_ls", "llama", "bf16", 2, 256, 2, 512, 64, 100, 2, 0, "dy", 3109), 45, 2, 16, 30, 0.1),
    "llama_rows": (Workload("opt_lr", "llama", "bf16", 2, 256, 4, 512, 64, 260, 16, 0, "dy", 3110), 65, 3, 16, 40, 0.0),
}
SEED, OFFSET, SITE = 77, 123456789012, 6


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def options(torch, st, case, seed=1):
    w, window, sinks, nb, R, p = case
    rng = np.random.default_rng(seed)
    table = bucket = g = None
    if nb:
        table = rng.standard_normal((nb, w.n_heads)).astype(np.float32)
        bucket = rng.integers(0, nb, 2 * R + 1).astype(np.int32)
        g = torch.zeros(nb, w.n_heads, device=st.dev)
    st.set_attention(window, sinks, None if table is None else st.f32(table),
                     None if bucket is None else torch.from_numpy(bucket).to(st.dev), g)
    if p:
        st.set_dropout(p, torch.tensor([SEED, OFFSET], dtype=torch.int64, device=st.dev), SITE)
    return table, bucket, g


def reference(case, inp, table, bucket):
    w, window, sinks, nb, R, p = case
    desc = oracle_desc(w)
    W, A = to64(inp, w)
    desc["score_add"] = score_add(w.seq, w.n_heads, w.arch == "llama", window, sinks, table, bucket)
    if p:
        for l, b in enumerate(W):
            b["keep_attn"] = keep(w.tokens, w.d_model, p, SEED, OFFSET, SITE + 2 * l)
            b["keep_ffn"] = keep(w.tokens, w.d_model, p, SEED, OFFSET, SITE + 2 * l + 1)
    y, caches = O.stage_forward(desc, W, A, inp["x"].astype(np.float64))
    return desc, W, A, y, caches


@pytest.mark.parametrize("name", sorted(CASES))
def test_stage_with_options_matches_the_oracle(torch, name):
    case = CASES[name]
    w = case[0]
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        table, bucket, g = options(torch, st, case)
        got = run_gpu(torch, st, w, inp, -1, want_dx=True)
        gt = None if g is None else g.cpu().numpy()
        # the terminator: nothing reaches block 0's attention
        if g is not None:
            g.zero_()
        cut = run_gpu(torch, st, w, inp, 0)
        gt0 = None if g is None else g.cpu().numpy()
    finally:
        st.close()
    desc, W, A, y, caches = reference(case, inp, table, bucket)
    dy = inp["dy"].astype(np.float64)
    dx, grads = O.stage_backward(desc, W, A, caches, dy, -1)
    # the stage's stated tolerances (1e-4 and 2e-2 of the largest element)
    chk = Checker("options_" + name, tol=1e-4 if w.dtype == "f32" else 2e-2)
    chk("y", got["y"], y)
    chk("dx", got["dx"], dx)
    single = w.placement == "ffn"
    chk.grads(got["grads"], [(None, b[1]) if single else b for b in grads], 0, w.n_blocks)
    if gt is not None:
        chk("table", gt, sum(table_grad(c["dscore"], case[3], bucket) for c in caches))
        chk("table_cut", gt0, table_grad(caches[1]["dscore"], case[3], bucket))
    chk.grads(cut["grads"], [(None, b[1]) if single else b for b in O.stage_backward(desc, W, A, caches, dy, 0)[1]],
              0, w.n_blocks)
    chk.done()


@pytest.mark.parametrize("name", ["bert_128", "llama", "f32"])
def test_options_off_again_leave_the_plain_stage(torch, name):
    case = CASES[name]
    w = case[0]
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        a = run_gpu(torch, st, w, inp, -1, want_dx=True)
        options(torch, st, case)
        b = run_gpu(torch, st, w, inp, -1, want_dx=True)
        st.set_attention()
        st.set_dropout(0.0)
        c = run_gpu(torch, st, w, inp, -1, want_dx=True)
    finally:
        st.close()
    assert not np.array_equal(a["y"], b["y"])
    assert np.array_equal(a["y"], c["y"]) and np.array_equal(a["dx"], c["dx"])
    for x, y in zip(a["grads"], c["grads"]):
        for u, v in zip(x, y):
            assert all(np.array_equal(u[k], v[k]) for k in u)


def test_a_window_over_everything_is_the_plain_attention(torch):
    """The same softmax by other kernels: equal within the roundings of P and O (two steps of bf16)."""
    case = CASES["llama"]
    w = case[0].replace(n_blocks=1)
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        a = run_gpu(torch, st, w, inp, 1)
        st.set_attention(window=10 ** 6)
        b = run_gpu(torch, st, w, inp, 1)
    finally:
        st.close()
    chk = Checker("window_all", tol=2e-2)
    chk("y", b["y"], a["y"])
    chk.done()


def test_options_are_refused_while_a_backward_is_pending_and_without_workspace(torch):
    w = CASES["bert_window"][0]
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        x, y = st.upload(inp["x"]), st.empty(*inp["x"].shape)
        rng = torch.zeros(2, dtype=torch.int64, device=st.dev)
        st.forward(x, y, 0)
        for call in (lambda: st.set_attention(window=3), lambda: st.set_dropout(0.1, rng)):
            with pytest.raises(B.RingadaError) as e:
                call()
            assert e.value.status == B.RINGADA_E_STATE
        st.backward(st.upload(inp["dy"]), 0)
        torch.cuda.synchronize()
        B.ringada_stage_set_attention(st.handle, B.StageAttention(window=3))
        with pytest.raises(B.RingadaError) as e:
            B.ringada_stage_forward(st.handle, st.sptr, x, y, w.batch, w.seq, 0, st.stash, st.stash_bytes, st.scratch,
                                    st.scratch_bytes)
        assert e.value.status == B.RINGADA_E_WORKSPACE
    finally:
        st.close()


def test_stage_with_options_in_a_graph(torch):
    """One captured iteration, replayed with new offsets, against eager iterations."""
    case = CASES["llama"]
    w = case[0]
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        options(torch, st, case)
        rng = st.rng
        x, y, dy, dx = st.upload(inp["x"]), st.empty(*inp["x"].shape), st.upload(inp["dy"]), st.empty(*inp["x"].shape)

        def step():
            st.zero_grads()
            st.forward(x, y, -1)
            st.backward(dy, -1, dx)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        seen = []
        for i in range(3):
            rng[1] = OFFSET + i
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (y, dx, st.adapters[0][0]["g_down"])]
            step()
            torch.cuda.synchronize()
            for a, b in zip(got, (y, dx, st.adapters[0][0]["g_down"])):
                assert torch.equal(a, b)
            seen.append(got[0])
        assert not torch.equal(seen[0], seen[1])
    finally:
        st.close()


def test_schedule_driver_with_dropout(torch):
    """Alg. 1's loop with a mask per iteration: the first iteration's loss and update against the oracle."""
    from paper_2502_19864_amd.schedule import Alg1Driver
    w = Workload("opt_sched", "bert", "f32", 2, 64, 2, 128, 16, 12, 3, 0, "cls_ce", 3120)
    inp = make_inputs(w)
    st = Stage(w, inp)
    try:
        drv = Alg1Driver(st, inp["w_h"], inp["b_h"], [(inp["x"], inp["labels"])], n_tm=2, lr=1.0, lr_head=0.01,
                         dropout=0.25, seed=9)
        rec = drv.run(d0=2, k=1, rounds=1, iters_per_round=1)
        wd = st.adapters[1][1]["w_down"].cpu().numpy()
    finally:
        st.close()
    desc = oracle_desc(w)
    W, A = to64(inp, w)
    for l, b in enumerate(W):
        b["keep_attn"], b["keep_ffn"] = (keep(w.tokens, w.d_model, 0.25, 9, 1, 2 * l + s) for s in (0, 1))
    ref, A2, _, _ = O.alg1_stage_run(desc, W, A, inp["w_h"].astype(np.float64), inp["b_h"].astype(np.float64),
                                     [(inp["x"].astype(np.float64), inp["labels"])], 2, 1, 2, 1, 1, 1, 1.0, 0.01)
    chk = Checker("schedule_dropout", tol=1e-4)
    chk("loss", np.array([rec[0]["loss"]]), np.array([ref[0][3]]))
    chk("update", wd - inp["adapters"][1][1]["w_down"], A2[1][1]["w_down"] - A[1][1]["w_down"])
    chk.done()
