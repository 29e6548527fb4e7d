"""Embedding of tokens, in 64 bits: rows of a table and their gradient, token by token."""
from __future__ import annotations

import numpy as np


def embed_fwd(ids, E, scale=1.0):
    """[*ids.shape, D]: scale * E[id], zeros where an id is outside the table."""
    V, D = E.shape
    Y = np.zeros(ids.shape + (D,))
    for at in np.ndindex(ids.shape):
        if 0 <= ids[at] < V:
            Y[at] = scale * E[ids[at]]
    return Y


def embed_bwd(ids, dY, V, scale=1.0, old=None):
    """old + scale * (the sums of dY's rows by token)."""
    D = dY.shape[-1]
    dE = np.zeros((V, D))
    for i, row in zip(ids.reshape(-1), dY.reshape(-1, D)):
        if 0 <= i < V:
            dE[i] += scale * row
    return dE if old is None else old + dE
