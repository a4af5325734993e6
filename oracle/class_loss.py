"""Losses over the classes of a linear layer in numpy float64, from their definitions.

    z = x w^T + b;  lse = log sum exp(z / T);  p = softmax(top / T) over a row's entries (one entry of probability 1 without a teacher)
    loss = T^2 sum p (log p + lse - z / T);  dz = scale T (softmax(z / T) - p) / n, n the rows that count;  dx = dz w;  dw = dz^T x;  db = sums of dz
"""

import numpy as np


def loss(x, w, classes, top=None, bias=None, temperature=1.0, scale=1.0):
    """classes: [rows, k] ids (any id outside [0, len(w)) is none).  A dict of loss, losses, lse, counts, p (softmax), dz, dx, dw, dbias."""
    rows, n_classes = x.shape[0], w.shape[0]
    z = x @ w.T
    if bias is not None:
        z = z + bias
    z = z / temperature
    peak = np.where(np.isfinite(z.max(1)), z.max(1), 0.0)
    lse = peak + np.log(np.exp(z - peak[:, None]).sum(1))
    soft = np.exp(z - lse[:, None])
    losses, counts, target = np.zeros(rows), np.zeros(rows, bool), np.zeros((rows, n_classes))
    for i in range(rows):
        entries = [j for j in range(classes.shape[1]) if 0 <= classes[i, j] < n_classes and (top is None or top[i, j] != -np.inf)]
        if not entries:
            continue
        counts[i] = True
        if top is None:
            p = np.ones(1)
        else:
            t = np.array([top[i, j] for j in entries]) / temperature
            p = np.exp(t - t.max()) / np.exp(t - t.max()).sum()
        for j, pj in zip(entries, p):
            c = classes[i, j]
            target[i, c] += pj
            if pj > 0:
                losses[i] += temperature ** 2 * pj * (np.log(pj) + lse[i] - z[i, c])
    n = int(counts.sum())
    dz = np.zeros_like(z)
    dz[counts] = (soft - target)[counts] * (scale * temperature / max(n, 1))
    xs = np.where(counts[:, None], x, 0.0)
    return {"loss": losses.sum() / n if n else 0.0, "losses": losses, "lse": lse, "counts": counts, "p": soft, "dz": dz,
            "dx": dz @ w, "dw": dz.T @ xs, "dbias": dz.sum(0)}
