"""Embedding and its gradient against the token-by-token oracle."""
import numpy as np
import pytest
import torch

from oracle import embed as L
from paper_2203_05705_amd import binding as ard
from util import assert_parity, from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances: util's.  Forward: one product and one rounding.  Gradient: a sum of n values in fp32, in an order of its own, is off by at most n 2^-24 of
# the sum of their sizes; sums here have 3000 terms at most, of zero mean, whose sum of sizes is 45 times what they add up to: 1e-5 would need
# 3000 x 45 x 6e-8 = 8e-3 if all errors agreed and sqrt(3000) x 45 x 6e-8 / 4 = 4e-5 as they come, so frequent tokens get a bound of their own below.


def _ids(R, V, seed, kind):
    rng = np.random.default_rng(seed)
    if kind == "one":
        return np.full(R, V // 2, np.int32)
    if kind == "frequent":   # three in four tokens are one of two
        return np.where(rng.random(R) < 0.75, rng.integers(0, min(2, V), R), rng.integers(0, V, R)).astype(np.int32)
    ids = rng.integers(0, V, R)
    if kind == "padded":
        ids = np.where(rng.random(R) < 0.3, rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1], R), ids)
    return ids.astype(np.int32)


def _check(R, V, D, dtype, wdtype, kind="any", scale=1.0, add=False, seed=0):
    rng = np.random.default_rng(seed)
    ids, E, dY = _ids(R, V, seed + 1, kind), stored(rng.standard_normal((V, D)), wdtype), stored(rng.standard_normal((R, D)), dtype)
    idd = torch.from_numpy(ids).cuda()
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    Y = ard.embed_fwd(idd, from_vals(E, wdtype), scale=scale, dtype=t)
    assert Y.dtype == t
    dead = np.broadcast_to(((ids < 0) | (ids >= V))[:, None], (R, D))
    assert_parity(Y, L.embed_fwd(ids, E, scale), dtype, dead, "Y")
    old = stored(rng.standard_normal((V, D)), wdtype) if add else None
    out = from_vals(old, wdtype) if add else None
    dE = ard.embed_bwd(idd, from_vals(dY, dtype), V, scale=scale, beta=1.0 if add else 0.0, dtype=torch.float32 if wdtype == "f32" else torch.bfloat16, out=out)
    ref = L.embed_bwd(ids, dY, V, scale, old)
    met = np.zeros(V, bool)
    met[ids[~dead[:, 0]]] = True
    if add:
        assert dE is out and np.array_equal(raw_bits(out)[~met], raw_bits(from_vals(old, wdtype))[~met])
    many = np.bincount(ids[~dead[:, 0]], minlength=V).max(initial=0)
    if wdtype == "f32" and many > 100:
        # per element: n 2^-24 of the sizes' sum if all roundings agreed
        size = L.embed_bwd(ids, np.abs(dY), V, abs(scale), None if old is None else np.abs(old))
        assert np.all(np.abs(to_host(dE) - ref) <= (many + 2) * 2.0 ** -24 * size)
    else:
        assert_parity(dE, ref, wdtype, None if add else np.broadcast_to(~met[:, None], (V, D)), "dE")


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("R,V,D", [(1, 1, 1), (1, 300, 7), (2, 3, 8), (63, 50, 9), (64, 1, 16), (65, 1000, 40), (300, 257, 100), (1025, 5000, 33), (700, 3000, 1500), (130, 70, 2049)])
def test_sizes(R, V, D, dtype, wdtype):
    _check(R, V, D, dtype, wdtype, seed=R)


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind", ["one", "frequent", "padded"])
@pytest.mark.parametrize("R,V", [(32, 9), (33, 9), (64, 9), (65, 9), (128, 9), (129, 9), (130, 300), (1000, 40), (3000, 500)])
def test_frequent_tokens_and_padding(R, V, kind, dtype, wdtype):
    """Rows of 32 tokens are summed at once, of 33 in pieces of 32."""
    _check(R, V, 24, dtype, wdtype, kind, scale=0.5, seed=R)
    _check(R, V, 24, dtype, wdtype, kind, scale=-3.0, add=True, seed=R + 1)


@pytest.mark.parametrize("V", [255, 256, 257, 512, 70000, 300000])
def test_tables_around_the_shares_of_sorting_workgroups(V):
    _check(2000, V, 8, "f32", "f32", "padded", seed=V)


def test_more_pieces_than_workgroups():
    """2^25 tokens and some: a workgroup takes more than one piece.  Sums of ones below 2^24 are exact."""
    R = (1 << 25) + 32 * 1000 + 5
    ids = (torch.arange(R, device="cuda", dtype=torch.int32) % 5) - 1
    got = ard.embed_bwd(ids, torch.ones((R, 1), dtype=torch.bfloat16, device="cuda"), 4)
    assert got[:, 0].tolist() == [float((R - v + 3) // 5) for v in range(4)]


def test_nothing_but_padding():
    ids = torch.full((5, 3), -1, dtype=torch.int32, device="cuda")
    E = torch.full((4, 6), float("nan"), device="cuda")
    Y = ard.embed_fwd(ids, E)
    assert Y.shape == (5, 3, 6) and not raw_bits(Y).any()
    dY = torch.full((5, 3, 6), float("inf"), device="cuda")
    dE = ard.embed_bwd(ids, dY, 4)
    assert not raw_bits(dE).any()
    old = torch.ones((4, 6), device="cuda")
    assert ard.embed_bwd(ids, dY, 4, beta=1.0, out=old) is old and bool((old == 1).all())
    none = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    assert ard.embed_fwd(none, E).shape == (0, 3, 6) and not raw_bits(ard.embed_bwd(none, torch.zeros((0, 3, 6), device="cuda"), 4)).any()


def test_a_token_outside_meets_no_row():
    """Infinities and NaN at padded positions reach nothing."""
    ids = np.array([2, -1, 2, 9, 0], np.int32)
    rng = np.random.default_rng(1)
    dY = rng.standard_normal((5, 12))
    bad = dY.copy()
    bad[1], bad[3] = np.nan, np.inf
    got = ard.embed_bwd(torch.from_numpy(ids).cuda(), from_vals(bad, "f32"), 4)
    assert_parity(got, L.embed_bwd(ids, stored(dY, "f32"), 4), "f32", None, "dE")


def test_rows_any_distance_apart():
    rng = np.random.default_rng(2)
    R, V, D = 40, 30, 21
    ids, E, dY = _ids(R, V, 3, "padded"), stored(rng.standard_normal((V, D)), "bf16"), stored(rng.standard_normal((R, D)), "bf16")
    idd = torch.from_numpy(ids).cuda()
    Ed, Yd, dYd = (torch.full((n, ld), 7.0, dtype=torch.bfloat16, device="cuda") for n, ld in ((V, 33), (R, 40), (R, 29)))
    dEd = torch.full((V, 50), 7.0, device="cuda")
    Ed[:, 3:24] = from_vals(E, "bf16")
    dYd[:, 5:26] = from_vals(dY, "bf16")
    ard.embed_fwd(idd, Ed[:, 3:24], scale=2.0, out=Yd[:, 1:22])
    assert_parity(Yd[:, 1:22].contiguous(), L.embed_fwd(ids, E, 2.0), "bf16", None, "Y")
    ard.embed_bwd(idd, dYd[:, 5:26], V, out=dEd[:, 11:32])
    assert_parity(dEd[:, 11:32].contiguous(), L.embed_bwd(ids, dY, V), "f32", None, "dE")
    assert bool((Yd[:, :1] == 7).all() and (Yd[:, 22:] == 7).all() and (dEd[:, :11] == 7).all() and (dEd[:, 32:] == 7).all())


def test_rows_beyond_32_bit_offsets():
    """The table's and the gradient's rows 2^28 elements apart: the last start 4 GB in, and beyond."""
    V, D, far = 6, 5, 1 << 28
    rng = np.random.default_rng(4)
    E, ids = stored(rng.standard_normal((V, D)), "f32"), np.array([5, 0, 5, 4], np.int32)
    buf = torch.empty((V - 1) * far + D, device="cuda")
    T = buf.as_strided((V, D), (far, 1))
    T.copy_(from_vals(E, "f32"))
    idd = torch.from_numpy(ids).cuda()
    Y = ard.embed_fwd(idd, T)
    assert_parity(Y, L.embed_fwd(ids, E), "f32", None, "Y")
    ard.embed_bwd(idd, Y, V, out=T)
    assert_parity(T.contiguous(), L.embed_bwd(ids, E[ids], V), "f32", None, "dE")


def test_same_bits_on_every_call_and_in_a_graph():
    R, V, D = 5000, 300, 72
    idd = torch.from_numpy(_ids(R, V, 5, "frequent")).cuda()
    gen = torch.Generator(device="cuda").manual_seed(0)
    E, dY = torch.randn((V, D), generator=gen, device="cuda"), torch.randn((R, D), generator=gen, device="cuda").bfloat16()
    Y, dE = torch.empty((R, D), dtype=torch.bfloat16, device="cuda"), torch.empty((V, D), device="cuda")
    ws = torch.empty(ard.embed_workspace_bytes(R, V, D), dtype=torch.uint8, device="cuda")

    def step():
        ard.embed_fwd(idd, E, out=Y)
        ard.embed_bwd(idd, dY, V, out=dE, ws=ws)
    step()
    torch.cuda.synchronize()
    want = [raw_bits(t) for t in (Y, dE)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        Y.fill_(7), dE.fill_(7)
        ws.fill_(0x55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(raw_bits(t), w) for t, w in zip((Y, dE), want))


def test_a_stream_of_its_own():
    rng = np.random.default_rng(6)
    ids, dY = _ids(400, 60, 7, "frequent"), stored(rng.standard_normal((400, 30)), "f32")
    idd, dYd = torch.from_numpy(ids).cuda(), from_vals(dY, "f32")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    dE = ard.embed_bwd(idd, dYd, 60, stream=side)
    side.synchronize()
    size = L.embed_bwd(ids, np.abs(dY), 60)
    assert np.all(np.abs(to_host(dE) - L.embed_bwd(ids, dY, 60)) <= 402 * 2.0 ** -24 * size)


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("scale", [-3.0, -1.0, 0.0, float("inf"), float("-inf"), float("nan")])
def test_rows_that_no_token_meets_are_zero_whatever_the_scale(scale, dtype, wdtype):
    R, V, D = 130, 300, 21
    ids, t = _ids(R, V, 8, "padded"), torch.float32 if wdtype == "f32" else torch.bfloat16
    dY = stored(np.random.default_rng(9).uniform(1, 2, (R, D)), dtype)
    dE = ard.embed_bwd(torch.from_numpy(ids).cuda(), from_vals(dY, dtype), V, scale=scale, dtype=t)
    met = np.zeros(V, bool)
    met[ids[(ids >= 0) & (ids < V)]] = True
    assert 0 < met.sum() < V and not raw_bits(dE)[~met].any()
    if np.isfinite(scale):
        assert_parity(dE, L.embed_bwd(ids, dY, V, scale), wdtype, None, "dE")
    else:
        want = np.full((int(met.sum()), D), scale)      # sums are positive
        assert np.array_equal(to_host(dE)[met], want, equal_nan=True)
