"""Layer norm over the rows of a matrix and its gradients, in 64 bits."""
from __future__ import annotations

import numpy as np


def layer_norm_fwd(X, gamma=None, beta=None, eps=1e-5):
    """(Y, mean, rstd) of X[R, D]."""
    mean = X.mean(axis=1)
    d = X - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    Y = d * rstd[:, None]
    if gamma is not None:
        Y = Y * gamma
    if beta is not None:
        Y = Y + beta
    return Y, mean, rstd


def layer_norm_bwd(dY, X, gamma, mean, rstd):
    """(dX, dgamma, dbeta)."""
    xh = (X - mean[:, None]) * rstd[:, None]
    q = dY if gamma is None else dY * gamma
    dX = rstd[:, None] * (q - q.mean(axis=1)[:, None] - xh * (q * xh).mean(axis=1)[:, None])
    return dX, (dY * xh).sum(axis=0), dY.sum(axis=0)
