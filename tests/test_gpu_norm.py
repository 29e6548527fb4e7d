"""Layer norm's kernels against the oracle: rows of every length class, both precisions, strided and compact rows."""
import numpy as np
import pytest
import torch

from oracle import norm as N
from paper_2203_05705_amd import binding as ard
from util import assert_parity, from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances: util's.  fp32 1e-5: a row's sums of up to 70000 terms are trees over lanes of short chains, a few 1e-7 of
# their terms' magnitude; rows here have offsets of the order of their spread, so centring costs no more.  The weight's
# gradients add up to 4097 rows in chains of at most a few hundred terms.  bf16: one rounding of each result.

DTYPES = [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")]


def _inputs(R, D, dtype, wdtype, seed):
    rng = np.random.default_rng(seed)
    X = stored(rng.standard_normal((R, D)) * (0.5 + rng.random((R, 1))) + 0.3 * rng.standard_normal((R, 1)), dtype)
    dY = stored(rng.standard_normal((R, D)), dtype)
    g, b = stored(1 + 0.3 * rng.standard_normal(D), wdtype), stored(0.3 * rng.standard_normal(D), wdtype)
    return X, dY, g, b


def _check(R, D, dtype, wdtype, seed, gamma=True, beta=True):
    X, dY, g, b = _inputs(R, D, dtype, wdtype, seed)
    g, b = g if gamma else None, b if beta else None
    Xd, dYd = from_vals(X, dtype), from_vals(dY, dtype)
    gd, bd = (None if w is None else from_vals(w, wdtype) for w in (g, b))
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd)
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    assert_parity(mean, rmean, "f32", None, "mean")
    assert_parity(rstd, rrstd, "f32", None, "rstd")
    assert_parity(Y, rY, dtype, None, "Y")
    dX, dg, db = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    rdX, rdg, rdb = N.layer_norm_bwd(dY, X, g, rmean, rrstd)
    if D > 2:   # (of one or two elements the gradient cancels to a rounding error of its terms)
        assert_parity(dX, rdX, dtype, None, "dX")
    else:
        assert np.max(np.abs(to_host(dX) - rdX)) <= 1e-5 * np.max(np.abs(dY)) * np.max(rrstd)
    assert (dg is None) == (db is None) == (not gamma)
    if gamma:
        if D > 1:
            assert_parity(dg, rdg, wdtype, None, "dgamma")
        assert_parity(db, rdb, wdtype, None, "dbeta")


@pytest.mark.parametrize("dtype,wdtype", DTYPES)
@pytest.mark.parametrize("R,D", [(1, 1), (3, 2), (5, 7), (4, 8), (2, 63), (9, 64), (3, 65), (7, 1000), (130, 1023), (6, 1024), (6, 1025), (1027, 1501),
                                 (5, 4095), (2, 4096), (3, 4097), (1, 16384)])
def test_rows_held_in_registers(R, D, dtype, wdtype):
    _check(R, D, dtype, wdtype, R * 7 + D)


@pytest.mark.parametrize("dtype,wdtype", DTYPES)
@pytest.mark.parametrize("R,D", [(1, 16385), (5, 20001), (67, 17000), (2, 70003)])
def test_rows_longer_than_registers(R, D, dtype, wdtype):
    _check(R, D, dtype, wdtype, R + D)


@pytest.mark.parametrize("R", [1, 2, 31, 33, 255, 511, 512, 513])
@pytest.mark.parametrize("D", [3, 8, 130, 300, 1000, 2049, 9000])
def test_few_rows(R, D):
    """One launch up to 512 rows, two from 513 on."""
    for dtype, wdtype in DTYPES:
        _check(R, D, dtype, wdtype, R + D)


@pytest.mark.parametrize("R,D", [(4097, 96), (2100, 1536), (300, 6000)])
def test_more_rows_than_workgroups(R, D):
    _check(R, D, "bf16", "f32", R)
    _check(R, D, "f32", "f32", R)


@pytest.mark.parametrize("D", [8, 127, 128, 129, 257, 384, 385, 520, 768, 769, 1026, 1535, 1537, 2100, 3071, 3080, 4100, 6144, 6145, 8200, 12288, 12290, 16383])
def test_rows_on_both_sides_of_every_number_of_runs(D):
    for R in (3, 520, 1030):
        _check(R, D, "bf16", "f32", R + D)
    _check(700, D, "bf16", "bf16", D)


# (not three elements: among 40007 such rows some lie so close together that mean and rstd rounded to fp32, all else exact, are 1.2e-4 off in dX)
@pytest.mark.parametrize("D", [4, 7, 8, 9, 31, 32, 33, 40, 63, 64, 65, 70, 128, 129])
def test_short_rows_several_a_wavefront(D):
    for R in (1, 5, 515, 1031, 40007):
        _check(R, D, "bf16", "f32", R + D)
        _check(R, D, "f32", "f32", R + D)
    _check(517, D, "bf16", "bf16", D)


@pytest.mark.parametrize("R,D", [(20001, 270), (8200, 600), (4099, 1101), (2051, 2177), (1027, 4353), (520, 8705)])
def test_enough_rows_for_more_elements_a_thread(R, D):
    _check(R, D, "bf16", "f32", R)
    _check(R, D, "bf16", "bf16", D)


@pytest.mark.parametrize("gamma,beta", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("D", [33, 2048, 18000])
def test_without_weights(gamma, beta, D):
    for dtype, wdtype in DTYPES:
        _check(6, D, dtype, wdtype, D, gamma, beta)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,D,shift", [(9, 37, 1), (70, 1024, 3), (5, 2001, 5), (3, 17000, 1)])
def test_rows_apart_from_each_other_at_any_element(dtype, R, D, shift, guarded_outputs):
    """Parts of the rows of wider matrices, starting at any element: nothing beside them is read or written."""
    X, dY, g, b = _inputs(R, D, dtype, dtype, D)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    wide = {}
    for name, vals in (("X", X), ("dY", dY)):
        wide[name] = torch.full((R, D + 2 * shift + 4), float("nan"), dtype=dt, device="cuda")
        wide[name][:, shift:shift + D] = from_vals(vals, dtype)
    gd, bd = from_vals(g, dtype), from_vals(b, dtype)
    Xv, dYv = wide["X"][:, shift:shift + D], wide["dY"][:, shift:shift + D]
    out = [guarded_outputs.tensor((R, D + shift + 5), dt) for _ in range(2)]
    before = [raw_bits(t) for t in out]
    Yv, dXv = out[0][:, shift:shift + D], out[1][:, shift:shift + D]
    Y, mean, rstd = ard.layer_norm_fwd(Xv, gd, bd, out=(Yv, None, None))
    dX, dg, db = ard.layer_norm_bwd(dYv, Xv, gd, mean, rstd, out=(dXv, guarded_outputs.tensor((D,), dt), guarded_outputs.tensor((D,), dt)))
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    rdX, rdg, rdb = N.layer_norm_bwd(dY, X, g, rmean, rrstd)
    for got, ref, what in ((Y, rY, "Y"), (dX, rdX, "dX"), (dg, rdg, "dgamma"), (db, rdb, "dbeta")):
        assert_parity(got.contiguous(), ref, dtype, None, what)
    for t, bits in zip(out, before):
        now = raw_bits(t)
        assert np.array_equal(now[:, :shift], bits[:, :shift]) and np.array_equal(now[:, shift + D:], bits[:, shift + D:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 8, 171, 683, 1029, 4097])
def test_compact_activations(dtype, D):
    """Kept units of a row pattern: the padding is not looked at and comes back as zeros."""
    R = 10
    X, dY, g, b = _inputs(R, D, dtype, "f32", D)
    pad = ard.pad8(D) - D
    Xd, dYd = (torch.nn.functional.pad(from_vals(t, dtype), (0, pad), value=float("nan")) for t in (X, dY))
    gd, bd = from_vals(g, "f32"), from_vals(b, "f32")
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd, D=D)
    dX, dg, db = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd, D=D)
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    rdX, rdg, rdb = N.layer_norm_bwd(dY, X, g, rmean, rrstd)
    assert_parity(Y[:, :D].contiguous(), rY, dtype, None, "Y")
    if D > 2:
        assert_parity(dX[:, :D].contiguous(), rdX, dtype, None, "dX")
        assert_parity(dg, rdg, "f32", None, "dgamma")
    assert_parity(db, rdb, "f32", None, "dbeta")
    assert not raw_bits(Y)[:, D:].any() and not raw_bits(dX)[:, D:].any()


@pytest.mark.parametrize("D", [5, 1024, 3000, 20000])
def test_rows_that_are_constant_or_hold_no_numbers(D):
    """A constant row gives beta; a NaN or an infinity stays in its row (and in the sums over rows of its columns)."""
    R = 6
    X, dY, g, b = _inputs(R, D, "f32", "f32", D)
    X[1] = 3.25
    Xd, dYd = from_vals(X, "f32"), from_vals(dY, "f32")
    Xd[3, D // 2], Xd[4, 0] = float("nan"), float("inf")
    gd, bd = from_vals(g, "f32"), from_vals(b, "f32")
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd)
    dX, dg, db = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    fine = [0, 1, 2, 5]
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    assert_parity(Y[fine].contiguous(), rY[fine], "f32", None, "Y")
    assert torch.equal(Y[1], bd)
    assert not torch.isfinite(Y[3]).any() and not torch.isfinite(Y[4]).any()
    rdX = N.layer_norm_bwd(dY, X, g, rmean, rrstd)[0]
    ordinary = [0, 2, 5]   # (the constant row's gradient is 1/sqrt(eps) times larger: on its own)
    assert_parity(dX[ordinary].contiguous(), rdX[ordinary], "f32", None, "dX")
    assert_parity(dX[1:2].contiguous(), rdX[1:2], "f32", None, "dX of a constant row")
    assert_parity(db, dY.sum(axis=0), "f32", None, "dbeta")


@pytest.mark.parametrize("rows", [50, 700])
def test_weights_gradients_one_at_a_time_and_none(rows):
    X, dY, g, b = _inputs(rows, 300, "bf16", "f32", 1)
    Xd, dYd, gd, bd = from_vals(X, "bf16"), from_vals(dY, "bf16"), from_vals(g, "f32"), from_vals(b, "f32")
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd)
    full = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    new = lambda: torch.empty(300, device="cuda")  # noqa: E731
    for out in ((None, new(), None), (None, None, new()), (None, None, None)):
        got = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd, out=out)
        for i in range(3):
            assert (got[i] is None) == (i > 0 and out[i] is None)
            assert got[i] is None or torch.equal(got[i], full[i])


@pytest.mark.parametrize("dtype,wdtype", DTYPES)
@pytest.mark.parametrize("R,D", [(1, 1), (40, 7), (70, 60), (130, 1000), (512, 2100), (513, 70), (1030, 1501), (700, 16384), (3, 17000), (130, 20001)])
def test_results_in_the_place_of_inputs(R, D, dtype, wdtype):
    """Y over X, dX over dY and over X: the bits of a call with results elsewhere."""
    X, dY, g, b = _inputs(R, D, dtype, wdtype, R + D)
    Xd, dYd, gd, bd = from_vals(X, dtype), from_vals(dY, dtype), from_vals(g, wdtype), from_vals(b, wdtype)
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd)
    want = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    over = Xd.clone()
    got = ard.layer_norm_fwd(over, gd, bd, out=(over, None, None))
    assert got[0] is over and all(torch.equal(p, q) for p, q in zip(got, (Y, mean, rstd)))
    for place in range(2):
        x, dy = Xd.clone(), dYd.clone()
        got = ard.layer_norm_bwd(dy, x, gd, mean, rstd, out=((dy, x)[place], torch.empty_like(gd), torch.empty_like(gd)))
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_same_bits_on_every_call_and_in_a_graph():
    X, dY, g, b = _inputs(2000, 1100, "bf16", "f32", 2)
    Xd, dYd, gd, bd = from_vals(X, "bf16"), from_vals(dY, "bf16"), from_vals(g, "f32"), from_vals(b, "f32")
    out = (torch.empty_like(Xd), torch.empty(2000, device="cuda"), torch.empty(2000, device="cuda"))
    grads = (torch.empty_like(Xd), torch.empty_like(gd), torch.empty_like(gd))
    ws = torch.empty(ard.layer_norm_workspace_bytes(2000, 1100), dtype=torch.uint8, device="cuda")

    def step():
        ard.layer_norm_fwd(Xd, gd, bd, out=out)
        ard.layer_norm_bwd(dYd, Xd, gd, out[1], out[2], out=grads, ws=ws)
    step()
    torch.cuda.synchronize()
    want = [raw_bits(t) for t in out + grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in out + grads:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(raw_bits(t), w) for t, w in zip(out + grads, want))


def test_a_stream_of_its_own():
    X, dY, g, b = _inputs(300, 515, "f32", "f32", 3)
    Xd, dYd, gd, bd = (from_vals(t, "f32") for t in (X, dY, g, b))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    Y, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd, stream=side)
    dX, dg, db = ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd, stream=side)
    side.synchronize()
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    assert_parity(Y, rY, "f32", None, "Y")
    assert_parity(dX, N.layer_norm_bwd(dY, X, g, rmean, rrstd)[0], "f32", None, "dX")


def test_rows_beyond_32_bit_offsets():
    """Three rows 2^30 elements apart: the last starts 4 GB into its buffer."""
    D, far = 72, 1 << 30
    buf = torch.empty(2 * far + D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(2 * far + D, dtype=torch.bfloat16, device="cuda")
    X, dY, g, b = _inputs(3, D, "bf16", "f32", 4)
    Xv, Yv = buf.as_strided((3, D), (far, 1)), out.as_strided((3, D), (far, 1))
    Xv.copy_(from_vals(X, "bf16"))
    gd, bd = from_vals(g, "f32"), from_vals(b, "f32")
    Y, mean, rstd = ard.layer_norm_fwd(Xv, gd, bd, out=(Yv, None, None))
    rY, rmean, rrstd = N.layer_norm_fwd(X, g, b)
    assert_parity(Y.contiguous(), rY, "bf16", None, "Y")
    dX, dg, db = ard.layer_norm_bwd(from_vals(dY, "bf16"), Xv, gd, mean, rstd, out=(Yv, torch.empty_like(gd), torch.empty_like(gd)))
    assert_parity(dX.contiguous(), N.layer_norm_bwd(dY, X, g, rmean, rrstd)[0], "bf16", None, "dX")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_of_very_long_rows(dtype):
    """A row of 2^25 elements.  A thread adds the sums of 2^13 (fp32) or 2^12 (bf16) runs, each with at most half an ulp of the growing sum, to
    either side: 2^6 halves of 2^-24, a thousandth of that once 1024 threads are added up, and 22 more roundings on the way there: 1.3e-6, of
    which the root halves the square sum's share.  2e-6 of each result; the mean's against the spread."""
    D = 1 << 25
    gen = torch.Generator(device="cuda").manual_seed(2)
    X, dY = (torch.randn((1, D), generator=gen, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16) for _ in range(2))
    dY += X   # (so that the mean of q xh is about 1)
    Y, mean, rstd = ard.layer_norm_fwd(X)
    dX, _, _ = ard.layer_norm_bwd(dY, X, None, mean, rstd)
    x, dy = to_host(X), to_host(dY)
    rY, rmean, rrstd = N.layer_norm_fwd(x)
    assert abs(to_host(mean)[0] - rmean[0]) * rrstd[0] <= 2e-6 and abs(to_host(rstd)[0] / rrstd[0] - 1) <= 2e-6
    rdX = N.layer_norm_bwd(dy, x, None, rmean, rrstd)[0]
    assert_parity(Y, rY, dtype, None, "Y")
    assert_parity(dX, rdX, dtype, None, "dX")
    if dtype == "f32":   # the kernel's mean of q xh, read off its result along xh
        xh = (x[0] - rmean[0]) * rrstd[0]
        assert abs((to_host(dX)[0] - rdX[0]) @ xh) / D <= 4e-6


def test_rows_of_more_columns_than_a_grid_has_threads_for():
    """2 x (2^25 + 24): the weights' gradients, 128 threads for each of their columns, at both ends and on both sides of the grid's limit."""
    R, D = 2, (1 << 25) + 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, dY = (torch.randn((R, D), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    g = 1 + 0.3 * torch.randn(D, generator=gen, device="cuda")
    Y, mean, rstd = ard.layer_norm_fwd(X, g)
    dX, dg, db = ard.layer_norm_bwd(dY, X, g, mean, rstd)
    x, dy, w = (to_host(t) for t in (X, dY, g))
    rY, rmean, rrstd = N.layer_norm_fwd(x, w)
    rdX, rdg, rdb = N.layer_norm_bwd(dy, x, w, rmean, rrstd)
    assert_parity(Y, rY, "bf16", None, "Y")
    assert_parity(dX, rdX, "bf16", None, "dX")
    assert_parity(dg, rdg, "f32", None, "dgamma")
    assert_parity(db, rdb, "f32", None, "dbeta")


def test_gradient_against_differences_of_the_forward_pass():
    """Along random directions: the change of sum(dY Y) in the oracle's 64 bits beside the kernel's gradients."""
    R, D = 5, 90
    X, dY, g, b = _inputs(R, D, "f32", "f32", 5)
    Xd, dYd, gd, bd = (from_vals(t, "f32") for t in (X, dY, g, b))
    _, mean, rstd = ard.layer_norm_fwd(Xd, gd, bd)
    grads = [to_host(t) for t in ard.layer_norm_bwd(dYd, Xd, gd, mean, rstd)]
    rng = np.random.default_rng(6)
    loss = lambda x, y, z: float((N.layer_norm_fwd(x, y, z)[0] * dY).sum())  # noqa: E731
    for i, at in enumerate((X, g, b)):
        way, args, h = rng.standard_normal(at.shape), [X, g, b], 1e-5
        args[i] = at + h * way
        up = loss(*args)
        args[i] = at - h * way
        diff, got = (up - loss(*args)) / (2 * h), float((grads[i] * way).sum())
        # (differences: h^2 of the third derivative and 1e-16 / h of rounding; the kernel: 1e-5 of its gradient's length)
        assert abs(diff - got) <= 2e-5 * np.linalg.norm(grads[i]) * np.linalg.norm(way) / np.sqrt(way.size) + 1e-6 * abs(diff)


@pytest.mark.parametrize("change,error", [(dict(dtype=7), -3), (dict(wdtype=1), -3), (dict(R=0), -2), (dict(D=0), -2), (dict(ldx=7), -2), (dict(ldy=7), -2),
                                          (dict(X=None), -1), (dict(mean=None), -1), (dict(eps=0.0), -1), (dict(flags=64), -1)])
def test_refusals(change, error):
    t = torch.zeros(64, device="cuda")
    a = dict(dtype=ard.F32, wdtype=ard.F32, R=4, D=8, X=t.data_ptr(), ldx=8, gamma=None, beta=None, eps=1e-5, Y=t.data_ptr(), ldy=8, mean=t.data_ptr(),
             rstd=t.data_ptr(), flags=0, stream=None)
    a.update(change)
    assert ard.lib().ard_layer_norm_fwd(*a.values()) == error and ard.lib().ard_last_error()
    torch.cuda.synchronize()
    assert not t.any()
