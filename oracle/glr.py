"""Gated linear recurrence, step by step in 64 bits:
c_t = s(f_t) c_{t-1} + (1 - s(f_t)) v_t,  h_t = s(o_t) c_t,  s the logistic function."""
from __future__ import annotations

import numpy as np


def sigmoid(x):
    with np.errstate(over="ignore"):
        return np.where(x >= 0, 1.0 / (1.0 + np.exp(-x)), np.exp(np.minimum(x, 0)) / (1.0 + np.exp(np.minimum(x, 0))))


def _live(T, B, lengths):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return np.arange(T)[:, None, None] < n[None, :, None]


def glr_fwd(f, v, o=None, c0=None, lengths=None):
    """(h, cT, states): f, v, o [T, B, H]; states [T + 1, B, H] with c0 first.  Behind a sequence's length its state stands
    and h is zero, whatever f, v and o hold there."""
    T, B, H = f.shape
    live = _live(T, B, lengths)
    f, v = np.where(live, f, 0.0), np.where(live, v, 0.0)
    states = np.zeros((T + 1, B, H))
    if c0 is not None:
        states[0] = c0
    for t in range(T):
        step = sigmoid(f[t]) * states[t] + sigmoid(-f[t]) * v[t]
        states[t + 1] = np.where(live[t], step, states[t])
    h = states[1:] if o is None else sigmoid(np.where(live, o, 0.0)) * states[1:]
    return np.where(live, h, 0.0), states[T], states


def glr_bwd(f, v, o, states, dh, dcT=None, lengths=None):
    """(df, dv, do, dc0); do is None without o."""
    T, B, H = f.shape
    live = _live(T, B, lengths)
    f, v, dh = (np.where(live, x, 0.0) for x in (f, v, dh))
    O = np.ones_like(f) if o is None else sigmoid(np.where(live, o, 0.0))
    df, dv, do = np.zeros_like(f), np.zeros_like(f), np.zeros_like(f)
    e = np.zeros((B, H)) if dcT is None else np.array(dcT, dtype=np.float64)
    for t in range(T - 1, -1, -1):
        F, I = sigmoid(f[t]), sigmoid(-f[t])
        dc = O[t] * dh[t] + e
        df[t] = np.where(live[t], dc * (states[t] - v[t]) * F * I, 0.0)
        dv[t] = np.where(live[t], dc * I, 0.0)
        do[t] = np.where(live[t], dh[t] * states[t + 1] * O[t] * (1 - O[t]), 0.0)
        e = np.where(live[t], F * dc, e)
    return df, dv, None if o is None else do, e
