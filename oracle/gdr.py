"""Gated delta rule, step by step in 64 bits: with a = s(f), w = s(b), kh = k / sqrt(|k|^2 + eps), qh likewise,
S_t = a S_{t-1} + w kh (v - a S_{t-1}^T kh)^T,  o_t = scale S_t^T qh.  Heads of v, f, b share those of q and k in groups."""
from __future__ import annotations

import numpy as np

from .glr import sigmoid


def _live(T, B, lengths):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return np.arange(T)[:, None] < n[None, :]


def _clean(live, *xs):
    return [np.where(live.reshape(live.shape + (1,) * (x.ndim - 2)), x, 0.0) for x in xs]


def _unit(x, eps):
    r = 1 / np.sqrt((x * x).sum(-1, keepdims=True) + eps)
    return x * r, r


def gdr_fwd(q, k, v, f, b, S0=None, lengths=None, scale=1.0, eps=1e-6):
    """(o, ST, states [T + 1, B, H, Dk, Dv] with S0 first).  Behind a sequence's length its state stands and o is zero."""
    T, B, Hk, Dk = q.shape
    H, Dv = v.shape[2:]
    live = _live(T, B, lengths)
    q, k, v, f, b = _clean(live, q, k, v, f, b)
    share = np.arange(H) // (H // Hk)
    qh, kh = _unit(q, eps)[0][:, :, share], _unit(k, eps)[0][:, :, share]
    states, o = np.zeros((T + 1, B, H, Dk, Dv)), np.zeros((T, B, H, Dv))
    if S0 is not None:
        states[0] = S0
    for t in range(T):
        a, w = sigmoid(f[t])[..., None, None], sigmoid(b[t])[..., None, None]
        faded = a * states[t]
        e = v[t] - np.einsum("bhij,bhi->bhj", faded, kh[t])
        S = faded + w * kh[t][..., None] * e[:, :, None, :]
        states[t + 1] = np.where(live[t][:, None, None, None], S, states[t])
        o[t] = np.where(live[t][:, None, None], scale * np.einsum("bhij,bhi->bhj", S, qh[t]), 0.0)
    return o, states[T], states


def gdr_bwd(q, k, v, f, b, states, do, dST=None, lengths=None, scale=1.0, eps=1e-6):
    """(dq, dk, dv, df, db, dS0)."""
    T, B, Hk, Dk = q.shape
    H, Dv = v.shape[2:]
    live = _live(T, B, lengths)
    q, k, v, f, b, do = _clean(live, q, k, v, f, b, do)
    share = np.arange(H) // (H // Hk)
    (qu, rq), (ku, rk) = _unit(q, eps), _unit(k, eps)
    qh, kh = qu[:, :, share], ku[:, :, share]
    dqh, dkh, dv, df, db = (np.zeros_like(x) for x in (qh, kh, v, f, b))
    dS = np.zeros((B, H, Dk, Dv)) if dST is None else np.array(dST, dtype=np.float64)
    for t in range(T - 1, -1, -1):
        on = live[t][:, None, None, None]
        a, w = sigmoid(f[t])[..., None, None], sigmoid(b[t])[..., None, None]
        faded = a * states[t]
        e = v[t] - np.einsum("bhij,bhi->bhj", faded, kh[t])
        d = dS + scale * qh[t][..., None] * do[t][:, :, None, :]
        dqh[t] = scale * np.einsum("bhij,bhj->bhi", states[t + 1], do[t])
        through = np.einsum("bhij,bhi->bhj", d, kh[t])
        de = w[..., 0] * through
        dkh[t] = w[..., 0] * np.einsum("bhij,bhj->bhi", d, e) - np.einsum("bhij,bhj->bhi", faded, de)
        dv[t] = de
        db[t] = (through * e).sum(-1) * sigmoid(b[t]) * sigmoid(-b[t])
        dfaded = d - kh[t][..., None] * de[:, :, None, :]
        df[t] = (dfaded * states[t]).sum((-1, -2)) * sigmoid(f[t]) * sigmoid(-f[t])
        dS = np.where(on, a * dfaded, dS)
    dqh, dkh, dv, df, db = _clean(live, dqh, dkh, dv, df, db)
    found = []
    for g, u, r in ((dqh, qu, rq), (dkh, ku, rk)):
        g = g.reshape(T, B, Hk, H // Hk, Dk).sum(3)
        found.append(r * (g - u * (u * g).sum(-1, keepdims=True)))
    return (*found, dv, df, db, dS)
