"""Loss against a teacher's largest logits and the labels, row by row in 64 bits."""
from __future__ import annotations

import numpy as np


def _softmax(x):
    m = x.max()
    e = np.exp(x - m)
    return e / e.sum(), m + np.log(e.sum())


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
                p, lse = _softmax(np.array([x for _, x in there]) / temperature)
                qT, zlse = _softmax(z / temperature)
                target = np.zeros(V)
                for (i, x), pk in zip(there, p):
                    target[i] += pk
                    if pk > 0:
                        loss[r] += alpha * temperature ** 2 * pk * ((x / temperature - lse) - (z[i] / temperature - zlse))
                dZ[r] += alpha * temperature * (qT - target)
        if alpha < 1 and labels is not None and 0 <= labels[r] < V:
            q, lse = _softmax(z)
            loss[r] += (1 - alpha) * (lse - z[labels[r]])
            q[labels[r]] -= 1
            dZ[r] += (1 - alpha) * q
        if dloss is not None:
            dZ[r] *= dloss[r]
    return loss, dZ
