"""The language model: embedding, norms, products, gated delta rule and distillation loss together, beside the same composition of
oracles; generation token by token; captured; training."""
import numpy as np
import pytest
import torch

from oracle import distill as DI
from oracle import embed as EM
from oracle import gdr as G
from oracle import norm as N
from paper_2203_05705_amd import binding as ard
from paper_2203_05705_amd import language as L
from util import raw_bits, to_host

pytestmark = pytest.mark.gpu

# fp32: util's 1e-5 of a single operator; two blocks of two norms' worth, two products and a recurrence, whose errors add up, pass the
# norms' factors (rows of an embedding scaled to length sqrt(D): near 1) and the unit keys (lengths above 1/2 here): ten times that.
CHAIN = 1e-4


def _close(got, ref, what):
    got = to_host(got)
    assert got.shape == ref.shape, what
    assert np.max(np.abs(got - ref)) <= CHAIN * np.max(np.abs(ref)), what


def _case(T, B, V, K, ragged, seed):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, V, (T, B)).astype(np.int32)
    top_ids = np.stack([rng.permutation(V)[:K] for _ in range(T * B)]).astype(np.int32)
    top, labels = rng.standard_normal((T * B, K)).astype(np.float32), rng.integers(0, V, T * B).astype(np.int32)
    n = None
    if ragged:
        n = np.array([T, 0, T // 3] + [T] * (B - 3), np.int32)
        behind = np.arange(T)[:, None] >= n[None]
        ids[behind] = -1
        top_ids[behind.reshape(-1)], labels[behind.reshape(-1)] = -1, -1
    return ids, top_ids, top, labels, n


def _oracle(model, ids, top_ids, top, labels, n, S0, dST, dloss):
    T, B = ids.shape
    w = [to_host(p) for p in model.params]
    E, blocks, gamma, beta = w[0], [w[i:i + 4] for i in range(1, len(w) - 2, 4)], w[-2], w[-1]
    cut, s, share = np.cumsum(model.parts)[:-1], model.Dk ** -0.5, model.D ** 0.5

    def parts(z):
        q, k, v, f, b = np.split(z.reshape(T, B, -1), cut, axis=-1)
        return q.reshape(T, B, model.Hk, -1), k.reshape(T, B, model.Hk, -1), v.reshape(T, B, model.H, -1), f, b
    x = EM.embed_fwd(ids, E, share).reshape(T * B, -1)
    kept, states = [], []
    for i, (g, c, W, Wy) in enumerate(blocks):
        nn, mean, rstd = N.layer_norm_fwd(x, g, c)
        p = parts(nn @ W.T)
        o, ST, every = G.gdr_fwd(*p, S0[i], n, s)
        kept.append((x, nn, mean, rstd, p, o, every))
        x = x + o.reshape(T * B, -1) @ Wy.T
        states.append(ST)
    nn, mean, rstd = N.layer_norm_fwd(x, gamma, beta)
    logits = nn @ E.T
    loss, dZ = DI.distill(logits, top_ids, top.astype(np.float64), labels, 2.0, 0.7, dloss)
    dE = dZ.T @ nn
    dx, dg, db = N.layer_norm_bwd(dZ @ E, x, gamma, mean, rstd)
    grads, dS0 = [dg, db], []
    for i in reversed(range(len(blocks))):
        g, _, W, Wy = blocks[i]
        x, nn, mean, rstd, p, o, every = kept[i]
        *dp, d0 = G.gdr_bwd(*p, every, (dx @ Wy).reshape(o.shape), dST[i], n, s)
        dz = np.concatenate([t.reshape(T * B, -1) for t in dp], axis=1)
        d, dg, db = N.layer_norm_bwd(dz @ W, x, g, mean, rstd)
        grads = [dg, db, dz.T @ nn, dx.T @ o.reshape(T * B, -1)] + grads
        dx = d + dx
        dS0 = [d0] + dS0
    return logits, states, loss, [EM.embed_bwd(ids, dx, model.V, share, dE)] + grads, dS0


@pytest.mark.parametrize("T,B,V,D,H,Hk,Dk,Dv", [(9, 4, 50, 24, 2, 1, 8, 12), (70, 3, 131, 40, 4, 2, 20, 16), (130, 3, 33, 64, 2, 2, 64, 64), (3, 5, 20, 16, 3, 1, 5, 7)])
@pytest.mark.parametrize("ragged", [False, True])
def test_forward_loss_and_gradients_against_the_oracles(T, B, V, D, H, Hk, Dk, Dv, ragged):
    model = L.Model(V, D, 2, H, Hk, Dk, Dv, torch.float32, seed=T)
    ids, top_ids, top, labels, n = _case(T, B, V, 6, ragged, T + 1)
    rng = np.random.default_rng(T + 2)
    S0, dST = (0.3 * rng.standard_normal((2, B, H, Dk, Dv)).astype(np.float32) for _ in range(2))
    dloss = (rng.random(T * B) / (T * B)).astype(np.float32)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    logits, states, saved = model.forward(dev(ids), dev(S0), dev(n))
    first = logits.clone()
    loss, _, dZ = ard.distill_fwd(logits, dev(top_ids), dev(top), labels=dev(labels), temperature=2.0, alpha=0.7, dloss=dev(dloss), out=(None, None, logits))
    assert dZ is logits
    grads, dS0 = model.backward(saved, dZ, dev(dST))
    want = _oracle(model, ids, top_ids, top, labels, n, S0.astype(np.float64), dST.astype(np.float64), dloss.astype(np.float64))
    _close(first, want[0], "logits")
    _close(loss, want[2], "loss")
    for i in range(2):
        _close(states[i], want[1][i], f"state {i}")
        _close(dS0[i], want[4][i], f"gradient of state {i}")
    assert len(grads) == len(want[3]) == len(model.params)
    for i, (got, ref) in enumerate(zip(grads, want[3])):
        _close(got, ref, f"gradient {i}")


def test_generation_follows_the_forward_pass():
    T, B, V = 70, 4, 90
    for dtype, tol in ((torch.float32, CHAIN), (torch.bfloat16, 2e-2)):   # bf16: values pass four bf16 stores a block (util.CEILING)
        model = L.Model(V, 64, 2, 4, 2, 16, 32, dtype, seed=3)
        ids = torch.from_numpy(np.random.default_rng(4).integers(0, V, (T, B)).astype(np.int32)).cuda()
        logits, states, _ = model.forward(ids)
        S, want = model.empty_state(B), logits.view(T, B, V).float()
        for t in range(T):
            assert (model.step(ids[t], S).float() - want[t]).abs().max() <= tol * want[t].abs().max()
        for a, b in zip(S, states):
            assert (a - b).abs().max() <= tol * b.abs().max()
        # a prompt at once, then one by one
        S = model.forward(ids[:66])[1]
        for t in range(66, T):
            assert (model.step(ids[t], S).float() - want[t]).abs().max() <= tol * want[t].abs().max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_and_replayed(dtype):
    T, B, V = 68, 3, 77
    model = L.Model(V, 48, 2, 2, 1, 16, 24, dtype, seed=5)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    cases = [[dev(a) for a in _case(T, B, V, 4, True, 6 + i)] for i in range(3)]

    def run(ids, top_ids, top, labels, n):
        logits, states, saved = model.forward(ids, lengths=n)
        loss, _, dZ = ard.distill_fwd(logits, top_ids, top, labels=labels, temperature=2.0, alpha=0.7, grad=True, out=(None, None, logits))
        return [loss, *states, *model.backward(saved, dZ)[0]]
    held = [t.clone() for t in cases[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(*held)
    for case in cases + cases[:1]:
        for t, value in zip(held, case):
            t.copy_(value)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, run(*case)):
            assert np.array_equal(raw_bits(got), raw_bits(want))


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 32), (torch.bfloat16, 8)])
def test_training_runs_and_repeats(dtype, bits):
    a, b = (L.train(6, T=20, B=4, V=60, D=32, K=4, dtype=dtype, bits=bits) for _ in range(2))
    assert a == b and len(a) == 6 and all(np.isfinite(a))
