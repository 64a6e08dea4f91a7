"""TEST INFRASTRUCTURE -- fp64 oracle of the preference loss of pairs of sequences.

lp_i = logits_i[label_i] - log sum exp logits_i for a counted row, L_s the sum over sequence s, and for a pair (c, r) with
the reference's sums R: m = beta ((L_c - R_c) - (L_r - R_r)), loss = -(1 - e) log sigma(m) - e log sigma(-m).
seqs: (first_row, len) of every sequence; pairs: (chosen, rejected, beta, e).
"""
from __future__ import annotations

from typing import Dict, Sequence, Tuple

import numpy as np


def _log_sigma(m: float) -> float:
    return -np.logaddexp(0.0, -m)


def _rows(logits, labels, seqs):
    V = logits.shape[1]
    for s, (first, n) in enumerate(seqs):
        for i in range(first, first + n):
            if 0 <= labels[i] < V:
                x = np.asarray(logits[i], dtype=np.float64)
                top = x.max()
                yield s, i, int(labels[i]), x - (top + np.log(np.exp(x - top).sum()))


def forward(logits, labels, seqs: Sequence[Tuple[int, int]], pairs, ref) -> Dict[str, np.ndarray]:
    row_logp, logp = np.zeros(logits.shape[0]), np.zeros(len(seqs))
    for s, i, y, lp in _rows(logits, labels, seqs):
        row_logp[i] = lp[y]
        logp[s] += lp[y]
    loss = np.zeros(len(pairs))
    for k, (c, r, beta, e) in enumerate(pairs):
        m = beta * ((logp[c] - ref[c]) - (logp[r] - ref[r]))
        loss[k] = (-(1.0 - e) * _log_sigma(m) if e < 1 else 0.0) + (-e * _log_sigma(-m) if e > 0 else 0.0)
    return {"row_logp": row_logp, "logp": logp, "loss": loss}


def backward(logits, labels, seqs, pairs, ref, dloss) -> np.ndarray:
    """dlogits of sum(loss * dloss)."""
    logp = forward(logits, labels, seqs, pairs, ref)["logp"]
    c_seq = np.zeros(len(seqs))
    for k, (c, r, beta, e) in enumerate(pairs):
        m = beta * ((logp[c] - ref[c]) - (logp[r] - ref[r]))
        slope = e * np.exp(_log_sigma(m)) - (1.0 - e) * np.exp(_log_sigma(-m))
        c_seq[c] += dloss[k] * beta * slope
        c_seq[r] -= dloss[k] * beta * slope
    in_pair = {s for c, r, _, _ in pairs for s in (c, r)}
    d = np.zeros(logits.shape)
    for s, i, y, lp in _rows(logits, labels, seqs):
        if s in in_pair:
            d[i] = -c_seq[s] * np.exp(lp)
            d[i, y] += c_seq[s]
    return d
