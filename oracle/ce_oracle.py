"""fp64 CPU oracle of the vocabulary projection's cross entropy.  TEST INFRASTRUCTURE ONLY.

For hidden rows H [T, d], a frozen projection W [d, vocab] and targets y (outside [0, vocab): the token has no loss):

    z_t = H_t . W,   lse_t = log sum_v exp(z_tv),   loss_t = lse_t - z_t,y(t)
    job_loss_j = sum_{t of j} w_t loss_t / sum_{t of j} w_t          (0 if the weights sum to 0)
    dH_t = g_t (softmax(z_t) - onehot(y_t)) . W^T,   g_t = w_t / sum w of its job, or the caller's

One numpy operation per line of the definition, rows without a loss are left out of every product.  Pinned by
tests/test_step_pins.py: torch autograd in float64, central differences, closed forms."""
from __future__ import annotations

import numpy as np


def cross_entropy(H, W, targets, offsets, weights=None, dloss=None):
    """dict of loss, lse [T], job_loss [J], dH [T, d], and for error bounds per row: P = g |softmax - onehot| and z."""
    H, W = np.asarray(H, dtype=np.float64), np.asarray(W, dtype=np.float64)
    T, V = H.shape[0], W.shape[1]
    y = np.asarray(targets, dtype=np.int64)
    live = np.flatnonzero((y >= 0) & (y < V))
    w = np.ones(T) if weights is None else np.asarray(weights, dtype=np.float64)
    loss, lse, share, dH = np.zeros(T), np.zeros(T), np.zeros(T), np.zeros_like(H)
    job_loss = np.zeros(len(offsets) - 1)
    z = H[live] @ W
    top = z.max(axis=1, keepdims=True) if len(live) else z
    lse[live] = top[:, 0] + np.log(np.exp(z - top).sum(axis=1)) if len(live) else 0
    loss[live] = lse[live] - z[np.arange(len(live)), y[live]]
    for j, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        mine = live[(live >= a) & (live < b)]
        total = w[mine].sum()
        if len(mine) and total != 0:
            share[mine] = w[mine] / total
            job_loss[j] = (share[mine] * loss[mine]).sum()
    g = share if dloss is None else np.where(np.isin(np.arange(T), live), np.asarray(dloss, dtype=np.float64), 0.0)
    P = np.exp(z - lse[live, None])
    P[np.arange(len(live)), y[live]] -= 1.0
    P *= g[live, None]
    dH[live] = P @ W.T
    return {"loss": loss, "lse": lse, "job_loss": job_loss, "dH": dH, "share": share, "live": live, "P": P, "z": z}
