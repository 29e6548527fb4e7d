"""The oracles of layer norm, the gated linear recurrence and AdamW pinned: gradients against central differences, the 8-bit
codes against their stated grids."""
import numpy as np
import pytest

from oracle import adamw as A
from oracle import glr as L
from oracle import norm as N


def _central(f, x, rng, n=12, h=1e-6):
    """[(index, central difference of f at x)] at n places."""
    flat = x.reshape(-1)
    got = []
    for i in rng.choice(flat.size, size=min(n, flat.size), replace=False):
        keep = flat[i]
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        down = f()
        flat[i] = keep
        got.append((i, (up - down) / (2 * h)))
    return got


@pytest.mark.parametrize("R,D", [(1, 1), (1, 5), (4, 2), (3, 17)])
@pytest.mark.parametrize("weights", [True, False])
def test_norm_gradients_are_those_of_the_forward_pass(R, D, weights):
    rng = np.random.default_rng(R * 100 + D)
    X, dY = rng.standard_normal((R, D)) + 0.5, rng.standard_normal((R, D))
    g, b = (1 + 0.3 * rng.standard_normal(D), rng.standard_normal(D)) if weights else (None, None)
    Y, mean, rstd = N.layer_norm_fwd(X, g, b)
    dX, dg, db = N.layer_norm_bwd(dY, X, g, mean, rstd)

    def loss():
        return float((N.layer_norm_fwd(X, g, b)[0] * dY).sum())
    # (differences of h = 1e-6 in 64 bits: truncation h^2 of third derivatives, which 1/eps = 1e5 bounds where a row is almost
    # constant, and 1e-16 / 1e-6 of rounding)
    for what, x in ((dX, X), (dg, g), (db, b)):
        if x is not None:
            for i, d in _central(loss, x, rng):
                assert abs(what.reshape(-1)[i] - d) <= 1e-5 * (1 + abs(d))


@pytest.mark.parametrize("T,B,H,gate,lengths", [(1, 1, 1, True, None), (5, 2, 3, True, None), (7, 3, 2, False, [0, 7, 4]), (6, 2, 2, True, [1, 6])])
def test_recurrence_gradients_are_those_of_the_forward_pass(T, B, H, gate, lengths):
    rng = np.random.default_rng(T)
    f, v, o, dh = (rng.standard_normal((T, B, H)) for _ in range(4))
    o = o if gate else None
    c0, dcT = rng.standard_normal((B, H)), rng.standard_normal((B, H))
    h, cT, states = L.glr_fwd(f, v, o, c0, lengths)
    df, dv, do, dc0 = L.glr_bwd(f, v, o, states, dh, dcT, lengths)

    def loss():
        h, cT, _ = L.glr_fwd(f, v, o, c0, lengths)
        return float((h * dh).sum() + (cT * dcT).sum())
    for what, x in ((df, f), (dv, v), (do, o), (dc0, c0)):
        if x is not None:
            for i, d in _central(loss, x, rng):
                assert abs(what.reshape(-1)[i] - d) <= 1e-7 * (1 + abs(d))


def test_nothing_behind_a_sequence_takes_part():
    rng = np.random.default_rng(1)
    f, v, o, dh = (rng.standard_normal((6, 3, 4)) for _ in range(4))
    lengths = [0, 3, 6]
    h, cT, states = L.glr_fwd(f, v, o, None, lengths)
    grads = L.glr_bwd(f, v, o, states, dh, None, lengths)
    for x in (f, v, o, dh):
        x[:, 0], x[3:, 1] = np.nan, np.inf
    h2, cT2, states2 = L.glr_fwd(f, v, o, None, lengths)
    for a, b in zip((h, cT) + grads, (h2, cT2) + L.glr_bwd(f, v, o, states2, dh, None, lengths)):
        assert np.array_equal(a, b)
    assert not h[:, 0].any() and not h[3:, 1].any() and not cT[0].any() and np.array_equal(cT[1], states[3, 1])


def test_logistic_function_over_its_range():
    x = np.array([-np.inf, -1e4, -50.0, -1.0, 0.0, 1.0, 50.0, 1e4, np.inf])
    assert np.allclose(L.sigmoid(x) + L.sigmoid(-x), 1.0) and np.all(np.diff(L.sigmoid(x)) >= 0)
    assert abs(L.sigmoid(np.array(-50.0)) - np.exp(-50)) < 1e-30


def test_adamw_first_step_and_decay():
    """After one step from zeros m / sqrt(v) is the gradient's sign whatever its size, so p moves by lr; without a gradient it
    decays by lr wd."""
    p, g = np.array([1.0, -2.0, 3.0]), np.array([1e-3, -7.0, 0.0])
    q, m, v = A.step(p, g, np.zeros(3), np.zeros(3), 0.1, 0.9, 0.999, 1e-12, 0.01, 1)
    assert np.allclose(q, p * (1 - 0.001) - 0.1 * np.sign(g), atol=1e-6)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)
    assert np.allclose(A.step(p, g, np.zeros(3), np.zeros(3), 0.1, 0.9, 0.999, 1e-12, 0.01, 1, scale=2.0)[1], 0.2 * g)


@pytest.mark.parametrize("n", [1, 255, 256, 257, 1000])
def test_codes_are_the_nearest_of_their_grids(n):
    rng = np.random.default_rng(n)
    m = (rng.standard_normal(n) * np.exp(3 * rng.standard_normal(n))).astype(np.float32)
    v = (m * m * rng.random(n).astype(np.float32)).astype(np.float32)
    (mc, mt), (vc, vt) = A.encode_m(m), A.encode_v(v)
    assert mc.dtype == np.int8 and vc.dtype == np.uint8 and mt.size == vt.size == -(-n // 256)
    mtop, vtop = np.repeat(mt, 256)[:n].astype(np.float64), np.repeat(vt, 256)[:n].astype(np.float64)
    # half a step on the grid of the root, and a little for the 32-bit roots
    assert np.max(np.abs(np.abs(mc) - 127 * np.sqrt(np.abs(m) / mtop))) <= 0.5 + 1e-4
    want = 255 * (v / vtop) ** 0.25
    assert np.max(np.abs(vc - np.where(v > 0, np.maximum(want, 1), 0))) <= 0.5 + 1e-4
    assert np.all(vc[v > 0] >= 1) and np.all((mc == 0) | (np.sign(mc) == np.sign(m)))
    # decoding: within a step's share of the values, and again the same codes
    dm, dv = A.decode_m(mc, mt), A.decode_v(vc, vt)
    assert np.max(np.abs(dm - m) / mtop) <= 1.0 / 127 + 1e-3
    assert np.array_equal(A.encode_m(dm)[0], mc) and np.array_equal(A.encode_v(dv)[0], vc)


def test_blocks_without_a_usable_scale():
    z = np.zeros(256, np.float32)
    for encode, decode in ((A.encode_m, A.decode_m), (A.encode_v, A.decode_v)):
        codes, top = encode(z)
        assert not codes.any() and not decode(codes, top).any()
        codes, top = encode(z + np.float32(1e-40))       # no reciprocal below the normal numbers
        assert not codes.any() and not decode(codes, top).any()
        for bad in (np.nan, np.inf):
            x = np.concatenate([z, z + np.float32(2)])
            x[3] = bad
            codes, top = encode(x)
            got = decode(codes, top)
            assert np.isnan(got[:256]).all() and np.allclose(got[256:], 2.0)


def test_states_in_8_bits_train_as_those_in_32():
    """A quadratic with curvatures over four orders of magnitude: both end near the minimum, at losses of one order."""
    rng = np.random.default_rng(0)
    n = 512
    scale, target = np.exp(rng.uniform(-4.6, 4.6, n)), rng.standard_normal(n)
    losses = {}
    for bits in (32, 8):
        p, m, v = np.zeros(n), np.zeros(n), np.zeros(n)
        for t in range(1, 401):
            g = scale * (p - target)
            p, m, v = A.step(p, g, m, v, 0.02, 0.9, 0.999, 1e-8, 0.0, t)
            if bits == 8:
                m, v = A.decode_m(*A.encode_m(m)).astype(np.float64), A.decode_v(*A.encode_v(v)).astype(np.float64)
        losses[bits] = float((scale * (p - target) ** 2).mean())
    start = float((scale * target ** 2).mean())
    assert losses[32] < 1e-2 * start and losses[8] < 2e-2 * start, (start, losses)
