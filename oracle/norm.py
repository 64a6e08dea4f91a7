"""TEST INFRASTRUCTURE -- fp64 oracle of the layer norm of a chunk-aligned batch, every task with its own weights.

Written row by row from the definition: y = (x - mean) / sqrt(var + eps) * gamma_t + beta_t with the mean and the variance
of the row; gradients by the chain rule through both.  X, dY: [T, N]; row_task: task of each row, -1 for padding (results
zero there); gamma, beta: per task [N] or None (ones, zeros).
"""
from __future__ import annotations

from typing import Dict, List, Optional

import numpy as np


def _weight(w, t: int, n: int, default: float) -> np.ndarray:
    return np.full(n, default) if w is None or w[t] is None else np.asarray(w[t], dtype=np.float64)


def forward(X, row_task, gamma, beta, eps: float) -> Dict[str, np.ndarray]:
    T, N = X.shape
    Y, mean, rstd = np.zeros((T, N)), np.zeros(T), np.zeros(T)
    for i in range(T):
        t = int(row_task[i])
        if t < 0:
            continue
        x = np.asarray(X[i], dtype=np.float64)
        mean[i] = x.sum() / N
        rstd[i] = 1.0 / np.sqrt(((x - mean[i]) ** 2).sum() / N + eps)
        Y[i] = (x - mean[i]) * rstd[i] * _weight(gamma, t, N, 1.0) + _weight(beta, t, N, 0.0)
    return {"Y": Y, "mean": mean, "rstd": rstd}


def backward(X, dY, row_task, n_tasks: int, gamma, eps: float) -> Dict[str, object]:
    T, N = X.shape
    dX = np.zeros((T, N))
    dg: List[np.ndarray] = [np.zeros(N) for _ in range(n_tasks)]
    db: List[np.ndarray] = [np.zeros(N) for _ in range(n_tasks)]
    for i in range(T):
        t = int(row_task[i])
        if t < 0:
            continue
        x, dy = np.asarray(X[i], dtype=np.float64), np.asarray(dY[i], dtype=np.float64)
        mean = x.sum() / N
        var = ((x - mean) ** 2).sum() / N
        s = 1.0 / np.sqrt(var + eps)
        h = dy * _weight(gamma, t, N, 1.0)
        dvar = (h * (x - mean)).sum() * -0.5 * s ** 3
        dmean = -(h * s).sum()                       # (the variance's own dependence on the mean sums to zero)
        dX[i] = h * s + dvar * 2.0 * (x - mean) / N + dmean / N
        dg[t] += dy * (x - mean) * s
        db[t] += dy
    return {"dX": dX, "dgamma": dg, "dbeta": db}
