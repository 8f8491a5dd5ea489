"""Oracle of the distillation loss on a teacher's top logits and of its gradient.  Test infrastructure: plain float64, row by
row from the definition

  p_j = softmax_j(t_j / tau) over entries with 0 <= idx_j < V,   q = softmax(z / tau),
  loss = tau^2 sum_j p_j (ln p_j - ln q_{idx_j}),   dz_v = w tau (q_v - sum_{j: idx_j = v} p_j);

p_j below 2^-126 of the largest, which fp32 holds as 0, has no term in the loss (on a class with q = 0 it would be infinite).
"""
from __future__ import annotations

import numpy as np


def _log_softmax(x):
    top = x.max()
    if top == -np.inf:
        return np.full(x.shape, np.nan)
    e = np.exp(x - top)
    with np.errstate(divide="ignore"):
        return x - top - np.log(e.sum())


def distill(z, idx, t, tau: float, weight=None):
    """(loss [rows], dz [rows, vocab], p [rows, top], ln q [rows, vocab]), float64."""
    z, t, idx = np.asarray(z, np.float64), np.asarray(t, np.float64), np.asarray(idx)
    R, V = z.shape
    loss, dz, ps, lqs = np.zeros(R), np.zeros((R, V)), np.zeros(t.shape), np.zeros((R, V))
    for r in range(R):
        lq = _log_softmax(z[r] / tau)
        lqs[r] = lq
        at = [j for j in range(idx.shape[1]) if 0 <= idx[r, j] < V]
        if not at or all(t[r, j] == -np.inf for j in at):
            continue
        lp = _log_softmax(t[r, at] / tau)
        w = 1.0 if weight is None else float(weight[r])
        dz[r] = w * tau * np.exp(lq)
        for j, l in zip(at, lp):
            p = np.exp(l)
            ps[r, j] = p
            if l - lp.max() >= -126 * np.log(2.0):
                loss[r] += tau * tau * p * (l - lq[idx[r, j]])
            dz[r, idx[r, j]] -= w * tau * p
    return loss, dz, ps, lqs
