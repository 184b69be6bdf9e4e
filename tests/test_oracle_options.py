"""Pins of the oracle's options (bias and window on the scores, dropout factors): central
differences of a small stage in float64, for every gradient they touch."""
import numpy as np
import pytest

import oracle as O
from paper_2502_19864_amd.workloads import Workload, make_inputs
from helpers import oracle_desc, to64
from stage_options import keep, score_add, table_grad

BUCKET = [3, 3, 2, 1, 0, 4, 5, 5, 5]  # R = 4


def build(arch, placement, table):
    w = Workload("opt", arch, "f32", 2, 16, 2, 24, 4, 7, 2, 0, "dy", 31, placement=placement)
    inp = make_inputs(w)
    desc = oracle_desc(w)
    W, A = to64(inp, w)
    for l, b in enumerate(W):
        b["keep_attn"] = keep(14, 16, 0.3, 5, 6, 2 * l)
        b["keep_ffn"] = keep(14, 16, 0.3, 5, 6, 2 * l + 1)
    desc["score_add"] = score_add(7, 2, arch == "llama", 3, 1, table, BUCKET)
    return w, inp, desc, W, A


@pytest.mark.parametrize("arch", ["bert", "llama"])
@pytest.mark.parametrize("placement", ["houlsby", "ffn"])
def test_gradients_with_options(arch, placement):
    rng = np.random.default_rng(3)
    table = rng.standard_normal((6, 2))
    w, inp, desc, W, A = build(arch, placement, table)
    x, dy = inp["x"].astype(np.float64), rng.standard_normal(inp["x"].shape)

    def loss(x=x, table=table, A=A):
        d = dict(desc, score_add=score_add(7, 2, arch == "llama", 3, 1, table, BUCKET))
        return float((O.stage_forward(d, W, A, x)[0] * dy).sum())

    y, caches = O.stage_forward(desc, W, A, x)
    dx, grads = O.stage_backward(desc, W, A, caches, dy, -1)
    dt = sum(table_grad(c["dscore"], 6, BUCKET) for c in caches)
    h = 1e-5

    def agree(got, plus, minus):  # truncation h^2, cancellation 1e-16 |loss| / h
        diff = (plus - minus) / (2 * h)
        assert abs(got - diff) <= 1e-6 * max(1.0, abs(diff)), (got, diff)

    u = rng.standard_normal(x.shape)
    agree((dx * u).sum(), loss(x=x + h * u), loss(x=x - h * u))
    u = rng.standard_normal(table.shape)
    agree((dt * u).sum(), loss(table=table + h * u), loss(table=table - h * u))
    for l in range(2):
        for a in range(2):
            if grads[l][a] is None:
                continue
            for k in ("w_down", "w_up"):
                u = rng.standard_normal(A[l][a][k].shape)

                def moved(s):
                    B = [list(p) for p in A]
                    B[l][a] = dict(A[l][a], **{k: A[l][a][k] + s * u})
                    return loss(A=B)
                agree((grads[l][a][k] * u).sum(), moved(h), moved(-h))
