"""The oracle's side of a stage's options: the scores' bias and mask, the table's gradient
and the dropout factors, written out from their definitions."""
import numpy as np

from operator_reference import philox


def score_add(S, H, causal, window=0, sinks=0, table=None, bucket=None):
    """[H, S, S]: the bias, -inf outside the window."""
    p, j = np.arange(S)[:, None], np.arange(S)[None, :]
    add = np.zeros((H, S, S))
    if table is not None:
        R = len(bucket) // 2
        add = add + np.transpose(np.asarray(table, np.float64)[np.asarray(bucket)[np.clip(j - p, -R, R) + R]], (2, 0, 1))
    if window:
        add = np.where((np.abs(p - j) < window) | (j < sinks), add, -np.inf)
    return add


def table_grad(dscore, n_buckets, bucket):
    """Sums of [B, H, S, S] over the pairs of each bucket: [n_buckets, H]."""
    S, R = dscore.shape[-1], len(bucket) // 2
    rel = np.arange(S)[None, :] - np.arange(S)[:, None]
    at = np.asarray(bucket)[np.clip(rel, -R, R) + R]
    d = dscore.sum(0)
    return np.array([[d[h][at == t].sum() for h in range(d.shape[0])] for t in range(n_buckets)])


def keep(T, d, p, seed, offset, site):
    """[T, d] factors of dropout."""
    thr = int(65536 * p + 0.5)
    u = np.array(philox(T * d, seed, offset, site)).reshape(T, d)
    return (u >= thr) * (65536 / (65536 - thr))
