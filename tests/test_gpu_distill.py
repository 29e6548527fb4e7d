"""The distillation loss and its gradient against the row-by-row oracle."""
import numpy as np
import pytest
import torch

from oracle import distill as L
from paper_2203_05705_amd import binding as ard
from util import assert_parity, from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances: util's.  An exponential of x is off by |x| 2^-24 + 2^-23 of itself, where |x| < 15 for all that counts in a sum: below 2e-6; the sums'
# own roundings, of positive terms in chains of at most 64 and trees, add below 1e-6.  fp32 1e-5, bf16 one rounding of each result.


def _case(R, V, K, dtype, tdtype, seed, labels=True):
    rng = np.random.default_rng(seed)
    Z, t = stored(2 * rng.standard_normal((R, V)), dtype), stored(2 * rng.standard_normal((R, K)), tdtype)
    ids = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(R)]).astype(np.int32).reshape(R, K)
    y = np.where(rng.random(R) < 0.2, rng.choice([-1, V, -2 ** 31], R), rng.integers(0, V, R)).astype(np.int32) if labels else None
    return Z, ids, t, y, rng.standard_normal(R).astype(np.float32).astype(np.float64)


def _run(Z, ids, t, y, dloss, dtype, tdtype, T, alpha):
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    Zd, td = from_vals(Z, dtype), from_vals(t, tdtype)
    args, kw = (dev(ids), td), dict(labels=dev(y), temperature=T, alpha=alpha)
    dl = from_vals(dloss, "f32")
    loss, stats, dZ = ard.distill_fwd(Zd, *args, dloss=dl, **kw)
    alone, stats2, none = ard.distill_fwd(Zd, *args, **kw)
    assert none is None and torch.equal(alone, loss) and torch.equal(stats, stats2)
    back = ard.distill_bwd(Zd, *args, stats, dl, **kw)
    assert np.array_equal(raw_bits(back), raw_bits(dZ))     # from the statistics: the same bits
    place = Zd.clone()
    assert ard.distill_fwd(place, *args, dloss=dl, out=(None, None, place), **kw)[2] is place and np.array_equal(raw_bits(place), raw_bits(dZ))
    place = Zd.clone()
    assert ard.distill_bwd(place, *args, stats, dl, out=place, **kw) is place and np.array_equal(raw_bits(place), raw_bits(dZ))
    return loss, dZ


def _check(R, V, K, dtype="f32", tdtype="f32", T=1.0, alpha=1.0, seed=0, case=None):
    Z, ids, t, y, dloss = case or _case(R, V, K, dtype, tdtype, seed)
    loss, dZ = _run(Z, ids, t, y, dloss, dtype, tdtype, T, alpha)
    rloss, rdZ = L.distill(Z, ids, t, y, T, alpha, dloss)
    assert_parity(loss, rloss, "f32", None, "loss")
    assert_parity(dZ, rdZ, dtype, None, "dZ")


TYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")]


@pytest.mark.parametrize("dtype,tdtype", TYPES)
@pytest.mark.parametrize("T,alpha", [(1.0, 1.0), (1.0, 0.3), (2.0, 1.0), (3.0, 0.5), (0.5, 0.0)])
@pytest.mark.parametrize("R,V,K", [(1, 1, 1), (3, 2, 2), (7, 33, 5), (5, 1000, 20), (2, 4099, 64)])
def test_temperatures_and_labels(R, V, K, T, alpha, dtype, tdtype):
    _check(R, V, K, dtype, tdtype, T, alpha, seed=R + V)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [255, 256, 257, 16383, 16384, 16385, 32767, 32768, 32769, 65535, 65537, 131072, 131075, 200001])
def test_rows_around_what_registers_hold(V, dtype):
    _check(2, V, 9, dtype, "f32", 2.0, 0.5, seed=V)


@pytest.mark.parametrize("K", [1, 63, 64, 65, 255, 256, 257, 1023, 1024])
@pytest.mark.parametrize("V", [40, 700])
def test_entries_around_a_wavefronts(K, V):
    """V = 40 names every element many times."""
    _check(3, V, K, "f32", "f32", 1.5, 0.8, seed=K)


def test_no_entries_is_the_labels_cross_entropy():
    Z, _, _, y, dloss = _case(9, 77, 1, "f32", "f32", 3)
    dev = torch.from_numpy(y).cuda()
    loss, _, dZ = ard.distill_fwd(from_vals(Z, "f32"), None, None, labels=dev, alpha=0.0, dloss=from_vals(dloss, "f32"))
    rl, rd = L.distill(Z, None, None, y, 1.0, 0.0, dloss)
    assert_parity(loss, rl, "f32", None, "loss")
    assert_parity(dZ, rd, "f32", None, "dZ")
    z = torch.zeros((9, 0), device="cuda")
    again = ard.distill_fwd(from_vals(Z, "f32"), z.int(), z, labels=dev, alpha=0.0, grad=True)
    assert torch.equal(again[0], loss)
    assert_parity(again[2], L.distill(Z, None, None, y, 1.0, 0.0)[1], "f32", None, "dZ of dloss 1")
    nothing = ard.distill_fwd(from_vals(Z, "f32"), None, None, grad=True)
    assert not raw_bits(nothing[0]).any() and bool((nothing[2] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_and_rows_that_they_leave_empty(dtype):
    R, V, K = 8, 500, 12
    Z, ids, t, y, dloss = _case(R, V, K, dtype, "f32", 4)
    y[:] = 3
    Z[0] = -np.inf                              # no logit left
    Z[1, :] = -np.inf
    Z[1, 3], ids[1, :] = 1.0, 3                 # one left, all entries on it
    Z[2, 100:] = -np.inf
    ids[2] = np.arange(K)
    t[3] = -np.inf                              # no entry left
    ids[4] = -1
    ids[5, ::2], t[5, 1::4] = V, -np.inf
    Z[6] = np.where(np.arange(V) % 2 == 1, Z[6], np.float32(-3e38))  # a mask of a large value
    ids[6] = 2 * np.arange(K) + 1
    y[4], y[7] = -1, V
    Z = stored(Z, dtype)
    _check(R, V, K, dtype, "f32", 2.0, 0.6, case=(Z, ids, t, y, dloss))
    loss, dZ = _run(Z, ids, t, y, dloss, dtype, "f32", 2.0, 0.6)
    assert not raw_bits(loss)[[0, 4]].any() and bool((dZ[0] == 0).all()) and bool((dZ[4] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 2.0, 4.0, 0.75])
def test_rows_of_a_masks_lowest_value(dtype, T):
    """All logits at the type's lowest value are as good as equal ones; one that is not takes the row."""
    R, V, K = 4, 300, 6
    Z, ids, t, y, dloss = _case(R, V, K, dtype, "f32", 9)
    lowest = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    Z[0] = lowest
    Z[1] = lowest
    Z[1, 7], ids[1], y[1] = 3.0, 7, 7
    Z[2] = 2.0 ** 40
    Z[3, ::2] = lowest
    ids[3], y[3] = 2 * np.arange(K) + 1, 11
    y[0], t[0] = 5, lowest
    _check(R, V, K, dtype, "f32", T, 0.6, case=(Z, ids, t, y, dloss))


def test_a_nan_stays_in_its_row():
    R, V, K = 4, 3000, 5
    Z, ids, t, y, dloss = _case(R, V, K, "f32", "f32", 5)
    clean = _run(Z, ids, t, y, dloss, "f32", "f32", 2.0, 0.5)
    y[:] = 7
    Z[2, 1234] = np.nan
    loss, _, dZ = ard.distill_fwd(from_vals(Z, "f32"), torch.from_numpy(ids).cuda(), from_vals(t, "f32"), temperature=2.0, grad=True)
    assert bool(torch.isnan(loss[2])) and bool(torch.isnan(dZ[2]).all()) and bool(torch.isfinite(loss[[0, 1, 3]]).all()) and bool(torch.isfinite(dZ[[0, 1, 3]]).all())
    Z[2] = np.nan
    loss, _, dZ = ard.distill_fwd(from_vals(Z, "f32"), torch.from_numpy(ids).cuda(), from_vals(t, "f32"), temperature=2.0, grad=True)
    assert bool(torch.isnan(loss[2])) and bool(torch.isnan(dZ[2]).all()) and len(clean) == 2


def test_large_logits_keep_their_differences():
    rng = np.random.default_rng(6)
    Z = stored(1e4 + 3 * rng.standard_normal((5, 300)), "f32")
    ids, t = np.tile(np.arange(4, dtype=np.int32), (5, 1)), stored(-2e4 + rng.standard_normal((5, 4)), "f32")
    _check(5, 300, 4, case=(Z, ids, t, None, np.ones(5)))


def test_rows_any_distance_apart_and_any_alignment():
    Z, ids, t, y, dloss = _case(6, 101, 4, "bf16", "bf16", 7)
    buf, out = (torch.full((6, 120), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    buf[:, 3:104] = from_vals(Z, "bf16")
    args, kw = (torch.from_numpy(ids).cuda(), from_vals(t, "bf16")), dict(labels=torch.from_numpy(y).cuda(), temperature=2.0, alpha=0.5)
    loss, stats, dZ = ard.distill_fwd(buf[:, 3:104], *args, dloss=from_vals(dloss, "f32"), out=(None, None, out[:, 5:106]), **kw)
    rl, rd = L.distill(Z, ids, t, y, 2.0, 0.5, dloss)
    assert_parity(loss, rl, "f32", None, "loss")
    assert_parity(out[:, 5:106].contiguous(), rd, "bf16", None, "dZ")
    assert bool((out[:, :5] == 7).all() and (out[:, 106:] == 7).all())


def test_rows_beyond_32_bit_offsets():
    R, V, far = 3, 40, (1 << 31) + 8
    Z, ids, t, y, dloss = _case(R, V, 3, "bf16", "f32", 8)
    buf = torch.empty((R - 1) * far + V, dtype=torch.bfloat16, device="cuda")
    place = buf.as_strided((R, V), (far, 1))
    place.copy_(from_vals(Z, "bf16"))
    loss, _, dZ = ard.distill_fwd(place, torch.from_numpy(ids).cuda(), from_vals(t, "f32"), dloss=from_vals(dloss, "f32"), out=(None, None, place))
    rl, rd = L.distill(Z, ids, t, None, 1.0, 1.0, dloss)
    assert_parity(loss, rl, "f32", None, "loss")
    assert_parity(place.contiguous(), rd, "bf16", None, "dZ")


def test_a_graph_and_a_stream_of_its_own():
    Z, ids, t, y, dloss = _case(50, 900, 8, "bf16", "f32", 9)
    Zd, idd, td, yd, dl = from_vals(Z, "bf16"), torch.from_numpy(ids).cuda(), from_vals(t, "f32"), torch.from_numpy(y).cuda(), from_vals(dloss, "f32")
    kw = dict(labels=yd, temperature=2.0, alpha=0.5)
    out = (torch.empty(50, device="cuda"), torch.empty((50, 3), device="cuda"), torch.empty_like(Zd))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    own = ard.distill_fwd(Zd, idd, td, dloss=dl, stream=side, **kw)
    side.synchronize()
    want = [raw_bits(x) for x in own]
    ard.distill_fwd(Zd, idd, td, dloss=dl, out=out, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ard.distill_fwd(Zd, idd, td, dloss=dl, out=out, **kw)
    for _ in range(3):
        for x in out:
            x.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(raw_bits(x), w) for x, w in zip(out, want))


def test_gradient_against_differences_of_the_loss():
    Z, ids, t, y, dloss = _case(20, 60, 6, "f32", "f32", 10)
    _, dZ = _run(Z, ids, t, y, dloss, "f32", "f32", 2.0, 0.5)
    way, e = np.random.default_rng(11).standard_normal(Z.shape), 1e-5
    diff = ((L.distill(Z + e * way, ids, t, y, 2.0, 0.5)[0] - L.distill(Z - e * way, ids, t, y, 2.0, 0.5)[0]) * dloss).sum() / (2 * e)
    assert abs(diff - (to_host(dZ) * way).sum()) <= 1e-5 * np.abs(to_host(dZ) * way).sum() + 1e-8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,alpha", [(1.0, 0.5), (2.0, 0.5), (1.5, 0.5), (2.0, 1.0), (1.0, 0.0)])
@pytest.mark.parametrize("V", [70, 9000, 140000])
def test_a_row_without_entries_and_label_is_left_out_whatever_it_holds(V, T, alpha, dtype):
    R, K = 6, 5
    Z, ids, t, y, dloss = _case(R, V, K, dtype, "f32", 11)
    y[:] = 4
    y[1:5], ids[1:5] = -1, -1
    ids[4], t[4] = 3, -np.inf       # entries without a share
    clean = Z.copy()
    Z[1, ::3], Z[2, 7], Z[3, :], Z[4, 5] = np.nan, np.inf, np.nan, -np.inf
    args, kw = (torch.from_numpy(ids).cuda(), from_vals(t, "f32")), dict(labels=torch.from_numpy(y).cuda(), temperature=T, alpha=alpha)
    dl, place, Zd = from_vals(np.where(np.arange(R) == 4, np.nan, dloss), "f32"), from_vals(Z, dtype), from_vals(Z, dtype)
    rloss, rdZ = L.distill(clean, ids, t, y, T, alpha, dloss)
    loss, stats, dZ = ard.distill_fwd(Zd, *args, dloss=dl, **kw)
    for l, d in ((loss, dZ), (loss, ard.distill_bwd(Zd, *args, stats, dl, **kw)), ard.distill_fwd(place, *args, dloss=dl, out=(None, None, place), **kw)[::2]):
        assert not raw_bits(l)[1:5].any() and not raw_bits(d)[1:5].any()
        assert_parity(l, rloss, "f32", None, "loss")
        assert_parity(d, rdZ, dtype, None, "dZ")
