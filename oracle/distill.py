"""Loss against a teacher's largest logits and the labels, row by row in 64 bits."""
from __future__ import annotations

import numpy as np


def _softmax(x):
    """Shares and their logarithms, from differences to the largest (whose place alone would take all digits of a far row)."""
    with np.errstate(invalid="ignore"):
        x = x - x.max()
    e = np.exp(x)
    return e / e.sum(), x - np.log(e.sum())


def distill(Z, ids, t, labels=None, temperature=1.0, alpha=1.0, dloss=None):
    """(loss[R], dZ[R, V]) of alpha T^2 KL(softmax(t / T) | softmax(Z / T)) + (1 - alpha) cross entropy."""
    R, V = Z.shape
    loss, dZ = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        z = Z[r]
        if np.all(z == -np.inf):
            continue
        if alpha > 0 and ids is not None:
            there = [(i, x) for i, x in zip(ids[r], t[r]) if 0 <= i < V and x != -np.inf]
            if there:
                p, logp = _softmax(np.array([x for _, x in there]) / temperature)
                qT, logq = _softmax(z / temperature)
                target = np.zeros(V)
                for (i, _), pk, lp in zip(there, p, logp):
                    target[i] += pk
                    if pk > 0:
                        loss[r] += alpha * temperature ** 2 * pk * (lp - logq[i])
                dZ[r] += alpha * temperature * (qT - target)
        if alpha < 1 and labels is not None and 0 <= labels[r] < V:
            q, logq = _softmax(z)
            loss[r] -= (1 - alpha) * logq[labels[r]]
            q[labels[r]] -= 1
            dZ[r] += (1 - alpha) * q
        if dloss is not None:
            dZ[r] *= dloss[r]
    return loss, dZ
