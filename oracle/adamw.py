"""The AdamW step and the 8-bit form of its states.

``step`` is the formula in 64 bits.  ``states_f32`` is the states' part of it in 32 bits, each operation rounded, which is
what the 8-bit codes are defined from; ``encode_*`` and ``decode_*`` are the codes of blocks of 256 neighbouring elements."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256
F = np.float32


def step(p, g, m, v, lr, beta1, beta2, eps, weight_decay, t, scale=1.0):
    """(p, m, v) after step t = 1, 2, ..."""
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = (1 - lr * weight_decay) * p - lr / (1 - beta1 ** t) * m / (np.sqrt(v) / math.sqrt(1 - beta2 ** t) + eps)
    return p, m, v


def states_f32(g, m, v, beta1, beta2, scale=1.0):
    g, m, v = g.astype(F) * F(scale), m.astype(F), v.astype(F)
    return m * F(beta1) + g * F(1 - beta1), v * F(beta2) + (g * g) * F(1 - beta2)


def _blocks(x):
    """[blocks, 256], the last one filled up with zeros."""
    n = x.size
    return np.concatenate([x.reshape(-1), np.zeros(-n % BLOCK, x.dtype)]).reshape(-1, BLOCK)


def _share(top):
    """1 / top in 32 bits; 0 where top is below the smallest normal number or is no number."""
    with np.errstate(invalid="ignore"):
        ok = (top >= F(2.0 ** -126)) & np.isfinite(top)
    return np.where(ok, F(1) / np.where(ok, top, F(1)), F(0)).astype(F)


def encode_m(m):
    """(int8 codes of m's shape, scales): sign and the nearest of 127 even steps of sqrt(|m| / largest)."""
    b = _blocks(m.astype(F))
    top = np.abs(b).max(axis=1)   # (NaN where one is)
    inv = _share(top)[:, None]
    with np.errstate(invalid="ignore"):
        c = np.where(inv > 0, np.rint(np.sqrt(np.abs(b) * inv) * F(127)), 0)
        c = np.where(b < 0, -c, c)
    return c.reshape(-1)[:m.size].astype(np.int8).reshape(m.shape), top


def encode_v(v):
    """(uint8 codes, scales): the nearest of 255 even steps of (v / largest)^(1/4), 1 at least where v > 0."""
    b = _blocks(v.astype(F))
    top = b.max(axis=1)
    inv = _share(top)[:, None]
    with np.errstate(invalid="ignore"):
        c = np.rint(np.sqrt(np.sqrt(b * inv)) * F(255))
        c = np.where(inv > 0, np.where(b > 0, np.maximum(c, 1), c), 0)
    return c.reshape(-1)[:v.size].astype(np.uint8).reshape(v.shape), top


def decode_m(codes, top):
    with np.errstate(invalid="ignore"):
        t = _blocks(codes).astype(F) * F(1 / 127)
        return (t * np.abs(t) * top.astype(F)[:, None]).reshape(-1)[:codes.size].reshape(codes.shape)


def decode_v(codes, top):
    with np.errstate(invalid="ignore"):
        t = _blocks(codes).astype(F) * F(1 / 255)
        t = t * t
        return (t * t * top.astype(F)[:, None]).reshape(-1)[:codes.size].reshape(codes.shape)
