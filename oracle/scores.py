"""Oracle: what a row of class scores answers, and distillation from a teacher's top classes (test infrastructure only).

Plain loops over rows in fp64, from the definitions:

* p = softmax(a / T); the log probability of a class, log sum exp(a / T), the entropy -sum p log p, the rank of a
  class under the order (score descending, class ascending) and the first k classes of that order whose score is
  above -inf;
* the distillation loss of a row with label y and teacher's list (c_t, z_t):
      w (-log p1_y) + (1 - w) T^2 sum_t q_t (log q_t - log pT_{c_t}),
  p1 = softmax(a), pT = softmax(a / T), q the softmax of z / T over the list ('logits') or exp(z) ('log_probs'), and
  its first derivatives and second derivatives' diagonal by the scores.
"""
import math

import numpy as np


def log_softmax(a, T):
    """log softmax(a / T) of one row (fp64); -inf where the score is -inf."""
    z = np.asarray(a, dtype=np.float64) / T
    m = z.max()
    if m == -np.inf:
        return z
    z = z - m  # first, so that scores far from zero lose nothing to the logarithm
    return z - math.log(np.exp(z).sum())


def log_probs(F, T=1.0, labels=None, k=0):
    """dict of logp, rank, lse, entropy (n,) and top_id, top_logp (k, n) for F (n, d)."""
    F = np.asarray(F, dtype=np.float64)
    n, d = F.shape
    out = {"lse": np.zeros(n), "entropy": np.zeros(n), "logp": np.zeros(n), "rank": np.full(n, -1, dtype=np.int32),
           "top_id": np.full((k, n), -1, dtype=np.int32), "top_logp": np.full((k, n), -np.inf)}
    for i in range(n):
        a = F[i]
        lp = log_softmax(a, T)
        m = a.max()
        out["lse"][i] = -np.inf if m == -np.inf else m / T + math.log(np.exp((a - m) / T).sum())
        on = lp > -np.inf
        out["entropy"][i] = -(np.exp(lp[on]) * lp[on]).sum()
        order = np.lexsort((np.arange(d), -a))
        if labels is not None and 0 <= labels[i] < d:
            out["logp"][i] = lp[labels[i]]
            out["rank"][i] = int(np.nonzero(order == labels[i])[0][0])
        best = [j for j in order[:k] if a[j] > -np.inf]
        for t, j in enumerate(best):
            out["top_id"][t, i] = j
            out["top_logp"][t, i] = lp[j]
    return out


def teacher_probs(ids, vals, d, T, kind):
    """(q, log q) of one row's list; 0 and 0 at unused places and at values of -inf."""
    ids, vals = np.asarray(ids), np.asarray(vals, dtype=np.float64)
    used = (ids >= 0) & (ids < d)
    used[used] = vals[used] > -np.inf
    q, lq = np.zeros(len(ids)), np.zeros(len(ids))
    if not used.any():
        return q, lq
    lq[used] = log_softmax(vals[used], T) if kind == "logits" else vals[used]
    q[used] = np.exp(lq[used])
    return q, lq


def distill(F, t_id, t_val, T=1.0, w=0.0, labels=None, kind="logits"):
    """(loss (n,), g (n, d), h (n, d)) in fp64 for F (n, d) and lists t_id, t_val (k, n)."""
    F = np.asarray(F, dtype=np.float64)
    n, d = F.shape
    loss, g, h = np.zeros(n), np.zeros((n, d)), np.zeros((n, d))
    for i in range(n):
        q, lq = teacher_probs(t_id[:, i], t_val[:, i], d, T, kind)
        lpT = log_softmax(F[i], T)
        pT = np.exp(lpT)
        g[i] = (1.0 - w) * T * q.sum() * pT
        h[i] = (1.0 - w) * q.sum() * pT * (1.0 - pT)
        for t in np.nonzero(q > 0)[0]:
            c = t_id[t, i]
            loss[i] += (1.0 - w) * T * T * q[t] * (lq[t] - lpT[c])
            g[i, c] -= (1.0 - w) * T * q[t]
        if w > 0.0 and 0 <= labels[i] < d:
            lp1 = log_softmax(F[i], 1.0)
            p1 = np.exp(lp1)
            loss[i] -= w * lp1[labels[i]]
            g[i] += w * p1
            g[i, labels[i]] -= w
            h[i] += w * p1 * (1.0 - p1)
    return loss, g, h
