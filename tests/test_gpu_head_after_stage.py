"""A stage, a trained final norm and a vocabulary head: one training step of a masked or causal language model with the
library's calls alone, against the float64 oracle and the formulas."""
import numpy as np
import pytest

import oracle as O
from helpers import TOL, oracle_desc, rel_err, to64
from paper_2502_19864_amd.workloads import Workload, make_inputs

pytestmark = pytest.mark.gpu

STAGES = {  # the pre-RMS stages are bf16 alone
    "llama_bf16": Workload("llama_bf16", "llama", "bf16", 2, 256, 2, 384, 64, 70, 2, 0, "dy", 3102),
    "bert_f32": Workload("bert_f32", "bert", "f32", 2, 128, 2, 256, 16, 32, 4, 1, "dy", 3103),
    "bert_bf16": Workload("bert_bf16", "bert", "bf16", 2, 256, 4, 512, 64, 45, 3, 0, "dy", 3104)}


def reference(w, inp, c, gain, shift, emb, labels):
    """The step in float64: the stage by the oracle, what lies behind it by torch's autograd."""
    import torch
    desc = oracle_desc(w)
    W, A = to64(inp, w)
    y, caches = O.stage_forward(desc, W, A, inp["x"].astype(np.float64))
    Y, G, E = (torch.from_numpy(np.ascontiguousarray(a)).double().requires_grad_() for a in (y, gain, emb))
    S = torch.from_numpy(shift).double().requires_grad_()
    if w.arch == "llama":
        n = Y * (Y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * G
    else:
        f = Y - Y.mean(-1, keepdim=True)
        n = f * (f.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * G + S
    keep = torch.from_numpy(labels >= 0)
    logp = torch.log_softmax(n[keep] @ E.T, 1)
    loss = -logp.gather(1, torch.from_numpy(labels).long()[keep][:, None]).mean()
    loss.backward()
    dx, grads = O.stage_backward(desc, W, A, caches, Y.grad.numpy(), c)
    return dict(loss=loss.item(), gain=G.grad.numpy(), shift=None if S.grad is None else S.grad.numpy(), emb=E.grad.numpy(), dx=dx), grads


@pytest.mark.parametrize("below", [False, True])
@pytest.mark.parametrize("name", sorted(STAGES))
def test_a_step_of_a_stage_and_a_vocabulary_head(name, below):
    """below: the gradient of the stage's input is wanted too."""
    import torch

    from paper_2502_19864_amd import operators as ops
    from paper_2502_19864_amd.stage import Stage
    w = STAGES[name]
    inp, c, V = make_inputs(w), -1 if below else w.lowest_unfrozen, 500
    rng = np.random.default_rng(w.seed)
    t = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    rounded = lambda a: torch.from_numpy(a.astype(np.float32)).to(t).float().numpy()
    gain, shift = rounded(1 + 0.1 * rng.standard_normal(w.d_model)), rounded(0.1 * rng.standard_normal(w.d_model))
    emb = rounded(rng.standard_normal((V, w.d_model)) * w.d_model ** -0.5)
    labels = rng.integers(0, V, (w.batch, w.seq)).astype(np.int32)
    labels[rng.random(labels.shape) < (0.85 if w.arch == "bert" else 0.2)] = -100
    want, want_grads = reference(w, inp, c, gain, shift, emb, labels)

    rms = w.arch == "llama"
    st = Stage(w, inp)
    try:
        G, S, E = st.upload(gain), None if rms else st.upload(shift), st.upload(emb)
        lab = torch.from_numpy(labels).cuda()
        y = st.empty(w.batch, w.seq, w.d_model)
        st.zero_grads()
        st.forward(st.upload(inp["x"]), y, c)
        n, s, stats = ops.norm_forward(y, G, S, rms=rms, eps=1e-6)
        count = int((labels >= 0).sum())
        dloss = (lab >= 0).float() / count
        loss, _, dn, dE = ops.vocab_ce_train(n, E, lab, dloss)
        dG, dS = torch.zeros_like(G, dtype=torch.float32), torch.zeros_like(G, dtype=torch.float32)
        dy = ops.norm_backward(dn, s, G, stats, rms=rms, dgain=dG, dshift=None if rms else dS, out=dn)
        dx = st.empty(w.batch, w.seq, w.d_model) if below else None
        st.backward(dy, c, dx)
        got = dict(loss=loss.double().sum().item() / count, gain=dG, shift=None if rms else dS, emb=dE, dx=dx)
        grads = st.grads()
        got = {k: v.double().cpu().numpy() if isinstance(v, torch.Tensor) else v for k, v in got.items()}
    finally:
        st.close()

    # fp32: the stages' bound; bf16: a dozen roundings between the input and the furthest gradient, in the mean square
    def close(what, a, b):
        if w.dtype == "f32":
            assert rel_err(a, b) <= TOL["f32"], (what, rel_err(a, b))
        else:
            off = np.linalg.norm(a - b) / np.linalg.norm(b)
            assert off <= 12 * 2.0 ** -8, (what, off)
    assert abs(got["loss"] - want["loss"]) <= (TOL["f32"] if w.dtype == "f32" else 12 * 2.0 ** -8) * want["loss"]
    for k in ("gain", "shift", "emb", "dx"):
        assert (got[k] is None) == (want[k] is None), k
        if want[k] is not None:
            close(k, got[k], want[k])
    for l in range(max(c, 0), w.n_blocks):
        for a in range(2):
            for k in ("w_down", "w_up"):
                close((l, a, k), grads[l][a][k], want_grads[l][a][k])
