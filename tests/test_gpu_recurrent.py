"""The residual recurrent block: its forward and backward pass beside the same composition of oracles, generation step by
step, and training."""
import numpy as np
import pytest
import torch

from oracle import glr as L
from oracle import norm as N
from oracle import patterns as P
from paper_2203_05705_amd import binding as ard
from paper_2203_05705_amd import recurrent as R
from util import assert_parity, to_host

pytestmark = pytest.mark.gpu

# fp32: util's 1e-5 of a single operator; a chain of three products, a norm and a recurrence, whose errors add up and pass
# through the gates' slopes (below 1/4), is given ten times that.
CHAIN = 1e-4


def _close(got, ref, what):
    got = to_host(got)
    assert got.shape == ref.shape, what
    assert np.max(np.abs(got - ref)) <= CHAIN * np.max(np.abs(ref)), what


@pytest.mark.parametrize("dp,b", [(1, 1), (2, 1), (3, 2)])
@pytest.mark.parametrize("ragged", [False, True])
def test_forward_and_backward_against_the_oracles(dp, b, ragged):
    T, B, D, H = 21, 3, 40, 50
    block = R.Block(D, H, torch.float32, seed=1)
    rng = np.random.default_rng(2)
    x, dy = (rng.standard_normal((T, B, D)).astype(np.float32) for _ in range(2))
    keep = P.keep_list(P.row_mask(H, dp, b)) if dp > 1 else np.arange(H)
    pat = ard.Pattern.row(dp, b) if dp > 1 else None
    k = len(keep)
    c0, dcT = (rng.standard_normal((B, k)).astype(np.float32) for _ in range(2))
    n = np.array([T, 0, 7], np.int32) if ragged else None
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    y, cT, saved = block.forward(dev(x), pat, dev(c0), dev(n))
    dx, grads, dc0 = block.backward(saved, dev(dy), dev(dcT))

    w = {name: to_host(p) for name, p in zip(block.NAMES, block.params)}
    x, dy = x.astype(np.float64).reshape(T * B, D), dy.astype(np.float64).reshape(T * B, D)
    nn, mean, rstd = N.layer_norm_fwd(x, w["gamma"], w["beta"])
    z = [(nn @ w[name][keep].T).reshape(T, B, k) for name in ("Wf", "Wv", "Wo")]
    h, rcT, states = L.glr_fwd(*z, c0, n)
    ry = x + h.reshape(T * B, k) @ w["Wy"][:, keep].T
    _close(y.view(T * B, D), ry, "y")
    _close(cT, rcT, "state")
    dh = (dy @ w["Wy"][:, keep]).reshape(T, B, k)
    *dz, rdc0 = L.glr_bwd(*z, states, dh, dcT, n)
    dz = [t.reshape(T * B, k) for t in dz]
    dn = sum(t @ w[name][keep] for t, name in zip(dz, ("Wf", "Wv", "Wo")))
    rdx, rdg, rdb = N.layer_norm_bwd(dn, x, w["gamma"], mean, rstd)
    _close(dx.view(T * B, D), rdx + dy, "dx")
    _close(dc0, rdc0, "dc0")
    ref = dict(gamma=rdg, beta=rdb)
    for t, name in zip(dz, ("Wf", "Wv", "Wo")):
        ref[name] = np.zeros((H, D))
        ref[name][keep] = t.T @ nn
    ref["Wy"] = np.zeros((D, H))
    ref["Wy"][:, keep] = dy.T @ h.reshape(T * B, k)
    for name, g in zip(block.NAMES, grads):
        _close(g, ref[name], "gradient of " + name)


def test_generation_follows_the_forward_pass():
    T, B, D, H = 12, 4, 64, 96
    for dtype, tol in ((torch.float32, CHAIN), (torch.bfloat16, 2e-2)):   # bf16: values pass four bf16 stores (util.CEILING)
        block = R.Block(D, H, dtype, seed=3)
        pat = ard.Pattern.row(2, 2)
        x = torch.randn((T, B, D), device="cuda").to(dtype)
        y, cT, _ = block.forward(x, pat)
        c = torch.zeros((B, ard.kept_count(pat, H)), device="cuda")
        for t in range(T):
            got, want = block.step(x[t], c, pat), y[t]
            assert (got.float() - want.float()).abs().max() <= tol * want.float().abs().max()
        assert (c - cT).abs().max() <= tol * cT.abs().max()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,dp", [(torch.float32, 1), (torch.bfloat16, 2)])
def test_training_learns_the_averages(dtype, dp, bits):
    losses = R.train(150, T=32, B=16, D=32, H=128, dp=dp, dtype=dtype, bits=bits)
    assert np.all(np.isfinite(losses))
    first, last = np.mean(losses[:5]), np.mean(losses[-10:])
    assert last < 0.5 * first, (first, last)
