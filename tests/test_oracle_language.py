"""The oracles of the embedding, the gated delta rule and the distillation loss against differences, and against each other's
simplest cases."""
import numpy as np
import pytest

from oracle import distill as DI
from oracle import embed as EM
from oracle import gdr as G


def _differences(loss, x, grad, seed, e=1e-6):
    rng = np.random.default_rng(seed)
    for _ in range(3):
        way = rng.standard_normal(x.shape)
        d = (loss(x + e * way) - loss(x - e * way)) / (2 * e)
        # e^2 of the third derivative and 1e-16 / e of rounding, both of the order of the terms added up
        assert abs(d - (grad * way).sum()) <= 1e-6 * (1 + np.abs(grad * way).sum())


def test_embedding():
    rng = np.random.default_rng(0)
    E, ids = rng.standard_normal((7, 5)), np.array([[3, -1, 3], [6, 7, 0]], np.int32)
    Y = EM.embed_fwd(ids, E, 2.0)
    assert np.array_equal(Y[0, 0], 2 * E[3]) and not Y[0, 1].any() and not Y[1, 1].any()
    dY = rng.standard_normal(Y.shape)
    _differences(lambda x: (EM.embed_fwd(ids, x, 2.0) * dY).sum(), E, EM.embed_bwd(ids, dY, 7, 2.0), 1)


@pytest.mark.parametrize("lengths", [None, [9, 0, 4]])
def test_gated_delta_rule(lengths):
    rng = np.random.default_rng(2)
    T, B, Hk, H, Dk, Dv = 9, 3, 2, 4, 5, 3
    x = [rng.standard_normal(s) for s in ((T, B, Hk, Dk), (T, B, Hk, Dk), (T, B, H, Dv), (T, B, H), (T, B, H), (B, H, Dk, Dv))]
    do, dST = rng.standard_normal((T, B, H, Dv)), rng.standard_normal((B, H, Dk, Dv))

    def loss(*x):
        o, ST, _ = G.gdr_fwd(*x, lengths, 0.7)
        return (o * do).sum() + (ST * dST).sum()
    states = G.gdr_fwd(*x, lengths, 0.7)[2]
    grads = G.gdr_bwd(*x[:5], states, do, dST, lengths, 0.7)
    for i in range(6):
        _differences(lambda y: loss(*x[:i], y, *x[i + 1:]), x[i], grads[i], i)


def test_gated_delta_rule_writes_what_it_is_told():
    """Orthogonal keys, strong gates: each key's value is read back, and the last one written where a key comes again."""
    k = np.eye(4)[[0, 1, 2, 1]][:, None, None, :]
    v = np.arange(1.0, 9.0).reshape(4, 1, 1, 2)
    strong = np.full((4, 1, 1), 60.0)
    o, ST, _ = G.gdr_fwd(k, k, v, strong, strong, eps=1e-30)
    assert np.allclose(o, v) and np.allclose(ST[0, 0], [v[0, 0, 0], v[3, 0, 0], v[2, 0, 0], [0, 0]])


def test_distillation():
    rng = np.random.default_rng(3)
    R, V, K = 6, 11, 4
    Z, t = rng.standard_normal((R, V)), rng.standard_normal((R, K))
    ids = np.stack([rng.permutation(V)[:K] for _ in range(R)]).astype(np.int32)
    ids[1, 2], ids[2, 1], t[3, 0] = ids[1, 0], -1, -np.inf
    labels, dloss = np.array([0, 3, -1, 11, 5, 5]), rng.random(R)
    for T, alpha in ((1.0, 1.0), (2.0, 0.6), (0.5, 0.0)):
        loss, dZ = DI.distill(Z, ids, t, labels, T, alpha, dloss)
        _differences(lambda x: (DI.distill(x, ids, t, labels, T, alpha)[0] * dloss).sum(), Z, dZ, 4)
        assert alpha < 1 or np.all(loss >= 0)
    # a teacher that the logits agree with, over all elements
    every = np.tile(np.arange(V), (R, 1))
    loss, dZ = DI.distill(Z, every, Z, None, 3.0, 1.0)
    assert np.abs(loss).max() < 1e-12 and np.abs(dZ).max() < 1e-12
