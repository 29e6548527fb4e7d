"""The gated linear recurrence's kernels against the step-by-step oracle: lengths around the stretches that wavefronts take,
time cut over workgroups, sequences of unequal length, every layout."""
import numpy as np
import pytest
import torch

from oracle import glr as L
from paper_2203_05705_amd import binding as ard
from util import assert_parity, from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances: util's.  fp32 1e-5: a gate is an exponential and a reciprocal of 1 ulp each, whose argument's rounding costs
# |f| 2^-24 <= 1e-6 of exp(-f) for the gates drawn here; 1 - F keeps its digits, so the states of long memories (the errors of
# 1 / (1 - F) steps, each 1e-7 of (1 - F) v) stay within some 1e-7 of their size.  bf16: one rounding of each result.


def _inputs(T, B, H, dtype, gate, seed, spread=5.0):
    rng = np.random.default_rng(seed)
    f = stored(rng.standard_normal((T, B, H)) + spread * rng.random(H), dtype)
    v, o, dh = (stored(rng.standard_normal((T, B, H)), dtype) for _ in range(3))
    c0, dcT = (rng.standard_normal((B, H)).astype(np.float32).astype(np.float64) for _ in range(2))
    return f, v, o if gate else None, dh, c0, dcT


def _dev(x, dtype="f32"):
    return None if x is None else from_vals(x, dtype)


def _lengths(T, B, seed):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, T + 1, B)
    n[0] = 0
    if B > 1:
        n[1] = T
    if B > 2:
        n[2] = min(1, T)
    return n.astype(np.int32)


def _compare(dtype, ref, got, dead):
    for what, r, g in zip(("h", "cT", "df", "dv", "do", "dc0"), ref, got):
        assert (r is None) == (g is None), what
        if r is not None:
            state = what in ("cT", "dc0")
            assert_parity(g.contiguous(), r, "f32" if state else dtype, None if state else dead, what)


def _check(T, B, H, dtype, gate=True, ragged=False, start=True, seed=0):
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, gate, seed)
    n = _lengths(T, B, seed) if ragged else None
    if not start:
        c0 = dcT = None
    rh, rcT, states = L.glr_fwd(f, v, o, c0, n)
    rgrads = L.glr_bwd(f, v, o, states, dh, dcT, n)
    fd, vd, od, dhd = (_dev(x, dtype) for x in (f, v, o, dh))
    nd = None if n is None else torch.from_numpy(n).cuda()
    if n is not None:   # what lies behind a sequence has no part in anything
        for x in (fd, vd, od, dhd):
            if x is not None:
                for b in range(B):
                    x[n[b]:, b] = float("nan") if b % 2 else float("inf")
    h, cT, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0), nd)
    assert ckpt.shape == (-(-T // ard.GLR_CHUNK), B, H)
    grads = ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT), nd)
    dead = None if n is None else np.broadcast_to(np.arange(T)[:, None, None] >= n[None, :, None], (T, B, H))
    _compare(dtype, (rh, rcT) + rgrads, (h, cT) + grads, dead)
    assert_parity(ckpt, states[0:T:ard.GLR_CHUNK], "f32", None, "states kept")
    # (without kept states: the same results)
    h2, cT2, none = ard.glr_fwd(fd, vd, od, _dev(c0), nd, train=False)
    assert none is None and np.array_equal(raw_bits(h2), raw_bits(h)) and torch.equal(cT2, cT)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 64, 127, 128, 129, 200, 257])
def test_steps_around_the_stretches(T, dtype):
    _check(T, 3, 130, dtype, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H", [(1, 1), (1, 2), (2, 3), (5, 63), (1, 64), (3, 65), (2, 127), (2, 128), (1, 129), (4, 1001), (33, 24)])
def test_sequences_and_channels(B, H, dtype):
    _check(37, B, H, dtype, seed=B + H)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("start", [True, False])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_with_and_without_a_gate_and_a_state(T, gate, start, dtype):
    _check(T, 2, 70, dtype, gate=gate, start=start, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("T,B,H", [(1, 5, 20), (16, 4, 33), (35, 20, 50), (150, 7, 66), (700, 5, 12)])
def test_sequences_of_unequal_length(T, B, H, gate, dtype):
    _check(T, B, H, dtype, gate=gate, ragged=True, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("T,B,H", [(1, 70, 1), (9, 200, 2), (20, 33, 5), (65, 50, 22), (130, 9, 37), (600, 48, 22), (300, 130, 3)])
def test_several_sequences_in_a_wavefront(T, B, H, gate, dtype):
    """Few channels a sequence: neighbouring lanes belong to sequences of different lengths."""
    _check(T, B, H, dtype, gate=gate, ragged=True, seed=T + B)
    _check(T, B, H, dtype, gate=gate, ragged=False, seed=T + B + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,H,ragged", [(1000, 1, 10, False), (4099, 1, 130, False), (2500, 3, 64, True), (20000, 1, 3, False)])
def test_time_cut_over_workgroups(T, B, H, ragged, dtype):
    assert ard.glr_workspace_bytes(ard.F32 if dtype == "f32" else ard.BF16, T, B, H) > 0
    _check(T, B, H, dtype, ragged=ragged, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cut_time_makes_the_pairs_that_are_read(dtype):
    """Of the segments' pairs in the workspace, [segment][P, S][B][H], the forward pass leaves the last out and the backward pass the first."""
    T, B, H = 2500, 3, 64
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, 9)
    fd, vd, od, dhd = (_dev(x, dtype) for x in (f, v, o, dh))
    n = ard.glr_workspace_bytes(ard.F32 if dtype == "f32" else ard.BF16, T, B, H) // 4
    segs, none = n // (2 * B * H), 12345.0
    ws = torch.full((segs, 2 * B * H), none, device="cuda")
    assert segs > 2 and ws.numel() == n
    _, _, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0), ws=ws)
    assert not (ws[:-1] == none).any() and (ws[-1] == none).all()
    ws.fill_(none)
    ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT), ws=ws)
    assert not (ws[1:] == none).any() and (ws[0] == none).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,H", [(1, 3, 20), (40, 20, 70), (2500, 3, 64), (4099, 2, 37), (20000, 1, 130)])
def test_gradients_in_the_place_of_what_they_are_made_from(T, B, H, dtype):
    """dc0 over dcT, and df, dv, do over f, v, o as well: the bits of a call with results elsewhere, time cut or not."""
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, T)
    fd, vd, od, dhd = (_dev(x, dtype) for x in (f, v, o, dh))
    n = torch.from_numpy(_lengths(T, B, T)).cuda() if B > 2 else None
    h, cT, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0), n)
    want = ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT), n)
    e = _dev(dcT)
    got = ard.glr_bwd(fd, vd, od, dhd, ckpt, e, n, out=(None, None, None, e))
    assert got[3] is e and all(torch.equal(p, q) for p, q in zip(got, want))
    e, place = _dev(dcT), [t.clone() for t in (fd, vd, od)]
    got = ard.glr_bwd(*place, dhd, ckpt, e, n, out=(*place, e))
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    place = [t.clone() for t in (fd, vd)]
    for out in place:
        a, b = (out, vd) if out is place[0] else (fd, out)
        assert torch.equal(ard.glr_fwd(a, b, od, _dev(c0), n, out=(out, None, None))[0], h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [1, 6, 171, 500, 683])
@pytest.mark.parametrize("T", [1, 35])
def test_kept_units_of_a_row_pattern(T, H, dtype):
    """Compact channels, padded to 8 with zeros, which come back as zeros."""
    B = 4
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, H)
    n = _lengths(T, B, H)
    pad = ard.pad8(H) - H
    fd, vd, od, dhd = (torch.nn.functional.pad(_dev(x, dtype), (0, pad)) for x in (f, v, o, dh))
    nd = torch.from_numpy(n).cuda()
    h, cT, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0), nd, H=H)
    grads = ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT), nd, H=H)
    rh, rcT, states = L.glr_fwd(f, v, o, c0, n)
    rgrads = L.glr_bwd(f, v, o, states, dh, dcT, n)
    cut = lambda t: t[..., :H] if t.shape[-1] != H else t  # noqa: E731
    _compare(dtype, (rh, rcT) + rgrads, tuple(cut(t) for t in (h, cT) + grads), None)
    for t in (h,) + grads[:3]:
        assert not raw_bits(t)[..., H:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch_first", [False, True])
@pytest.mark.parametrize("H", [64, 37])
def test_parts_of_one_product_in_either_order(batch_first, H, dtype, guarded_outputs):
    """f, v, o as parts of the rows of one product, time or batch first; gradients into parts likewise, nothing beside them."""
    T, B = 50, 3
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, H)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    first, second = (B, T) if batch_first else (T, B)

    def view(t, at):
        t = t[..., at:at + H]
        return t.transpose(0, 1) if batch_first else t
    Z = torch.full((first, second, 3 * H + 5), float("nan"), dtype=dt, device="cuda")
    parts = [view(Z, 1 + i * (H + 1)) for i in range(3)]
    for p, x in zip(parts, (f, v, o)):
        p.copy_(_dev(x, dtype))
    D = torch.full((first, second, H + 3), float("nan"), dtype=dt, device="cuda")
    view(D, 2).copy_(_dev(dh, dtype))
    hO, dZ = guarded_outputs.tensor((first, second, H + 2), dt), guarded_outputs.tensor((first, second, 3 * H + 5), dt)
    before = [raw_bits(t) for t in (hO, dZ)]
    h, cT, ckpt = ard.glr_fwd(*parts, c0=_dev(c0), out=(view(hO, 1), None, None))
    grads = ard.glr_bwd(*parts, view(D, 2), ckpt, dcT=_dev(dcT), out=[view(dZ, 1 + i * (H + 1)) for i in range(3)])
    rh, rcT, states = L.glr_fwd(f, v, o, c0)
    _compare(dtype, (rh, rcT) + L.glr_bwd(f, v, o, states, dh, dcT), (h, cT) + grads, None)
    untouched = [[0, H + 1], [0, H + 1, 2 * H + 2, 3 * H + 3, 3 * H + 4]]
    for t, bits, cols in zip((hO, dZ), before, untouched):
        assert np.array_equal(raw_bits(t)[..., cols], bits[..., cols])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_at_the_ends_of_their_range(dtype):
    """Gates that are open or shut for good, infinite ones among them: F = 1 keeps the state exactly, F = 0 replaces it."""
    T, B, H = 40, 2, 8
    f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, 1)
    for k, x in enumerate((np.inf, -np.inf, 1e4, -1e4, 90.0, -90.0)):
        f[..., k] = x
        o[..., k] = -x
    f, o = stored(f, dtype), stored(o, dtype)
    fd, vd, od, dhd = (_dev(x, dtype) for x in (f, v, o, dh))
    h, cT, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0))
    grads = ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT))
    rh, rcT, states = L.glr_fwd(f, v, o, c0)
    _compare(dtype, (rh, rcT) + L.glr_bwd(f, v, o, states, dh, dcT), (h, cT) + grads, None)
    assert torch.equal(cT[:, 0], _dev(c0)[:, 0]) and torch.equal(cT[:, 1], vd[-1, :, 1].float())


@pytest.mark.parametrize("dtype,T,B,H", [("f32", 8192, 64, 256), ("f32", 32768, 1, 60), ("bf16", 32768, 64, 512), ("bf16", 32768, 2, 62), ("f32", 24, 3, 60)])
def test_long_memories_of_steady_gates(dtype, T, B, H):
    """Gates and inputs that stay as they are, where roundings of one sign would add up, against the closed form
    c_T = v + (c0 - v) F^T, e_0 = F^T e_T + dh F (1 - F^T) / (1 - F).  A state is rounded once in 8 steps, half an ulp to either side: 6 deviations
    of their sum; the gate's argument costs |f| 2^-24 of 1 - F and its operations 4 ulp."""
    code, dt = (ard.F32, torch.float32) if dtype == "f32" else (ard.BF16, torch.bfloat16)
    assert (ard.glr_workspace_bytes(code, T, B, H) > 0) == (T > 64 and B < 10)   # (time cut, and not)
    k = np.arange(H)
    f, v, c0 = np.array([8.0, 9, 10, 11, 12, 14])[k % 6], np.array([1.0, 0, -0.5])[k % 3], np.array([0.0, 1, 2, -1])[k % 4]
    dh, dcT = np.array([0.0, 1, -0.5])[k % 3], np.array([1.0, 0, 2, -1])[k % 4]
    fd, vd, dhd = (_dev(x, dtype).expand(T, B, H) for x in (f, v, dh))
    c0d, dcTd = (_dev(x).expand(B, H).contiguous() for x in (c0, dcT))
    h, cT, ckpt = ard.glr_fwd(fd, vd, None, c0d)
    df, dv, _, dc0 = ard.glr_bwd(fd, vd, None, dhd, ckpt, dcTd)
    I = L.sigmoid(-f)
    FT = np.exp(T * np.log1p(-I))
    rc, re = v + (c0 - v) * FT, FT * dcT + dh * (1 - I) * -np.expm1(T * np.log1p(-I)) / I
    tol = 2.0 ** -24 * (6 * np.sqrt(T / 8 / 3) + f + 4)
    bound_c, bound_e = tol * (np.abs(v) + np.abs(c0 - v)), tol * (np.abs(dcT) + np.abs(dh) * np.minimum(T, 1 / I))
    assert (np.abs(to_host(cT) - rc) <= bound_c).all()
    assert (np.abs(to_host(dc0) - re) <= bound_e).all()
    round_off = 1e-6 if dtype == "f32" else 2.0 ** -8
    assert (np.abs(to_host(h[-1]) - rc) <= bound_c + round_off * np.abs(rc)).all()
    dc = re / (1 - I)   # of the first step
    assert (np.abs(to_host(dv[0]) - dc * I) <= (bound_e + round_off * np.abs(dc) + tol * np.abs(dc)) * I).all()
    want = dc * (c0 - v) * I * (1 - I)
    assert (np.abs(to_host(df[0]) - want) <= bound_e * np.abs(c0 - v) * I + (round_off + tol) * np.abs(want)).all()


def test_long_memories_step_by_step():
    """The same by single steps, the state in its place: a rounding each."""
    T, B, H = 4096, 2, 60
    k = np.arange(H)
    f, v, c0 = np.array([8.0, 9, 10, 11, 12, 14])[k % 6], np.array([1.0, 0, -0.5])[k % 3], np.array([0.0, 1, 2, -1])[k % 4]
    fd, vd, c = _dev(f).expand(1, B, H), _dev(v).expand(1, B, H), _dev(c0).expand(B, H).contiguous()
    out = (torch.empty((1, B, H), device="cuda"), c, None)
    for _ in range(T):
        ard.glr_fwd(fd, vd, None, c, train=False, out=out)
    want = v + (c0 - v) * np.exp(T * np.log1p(-L.sigmoid(-f)))
    assert (np.abs(to_host(c) - want) <= 2.0 ** -24 * (6 * np.sqrt(T / 3) + f + 4) * (np.abs(v) + np.abs(c0 - v))).all()


@pytest.mark.parametrize("T", [1, 7, 40, 300, 5000])
def test_an_infinite_state_stays_one(T):
    f, v = (torch.full((T, 2, 8), x, device="cuda") for x in (3.0, 0.5))
    f[..., 4:] = float("inf")
    c0 = torch.zeros(2, 8, device="cuda")
    c0[0, ::2], c0[1, 1::2] = float("inf"), -float("inf")
    h, cT, _ = ard.glr_fwd(f, v, None, c0)
    inf = torch.isinf(c0)
    assert torch.equal(cT[inf], c0[inf]) and torch.isfinite(cT[~inf]).all()
    assert torch.equal(h[:, inf], c0[inf].expand(T, -1)) and torch.isfinite(h[:, ~inf]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 30, 700])
def test_gradients_of_gates_that_are_almost_open_or_shut(T, dtype):
    """df and do of f and o from -20 to 20, each element beside itself: 1 - s(x) of an x past 8 is smaller than the rounding of s(x).
    fp32: two gates' arguments, (|f| + |o|) 2^-24, some ten operations of 2^-24 and the state's 1e-6; bf16: its rounding, 2^-8 too."""
    B, H = 2, 41
    rng = np.random.default_rng(T)
    x = np.linspace(-20, 20, H)
    o = stored(np.broadcast_to(x, (T, B, H)), dtype)
    f = stored(np.broadcast_to(x[::-1], (T, B, H)), dtype)
    v, dh = (stored(0.5 + rng.random((T, B, H)), dtype) for _ in range(2))   # (positive: no element of a gradient is small by cancellation)
    c0 = stored(2.0 + rng.random((B, H)), "f32")
    h, cT, ckpt = ard.glr_fwd(_dev(f, dtype), _dev(v, dtype), _dev(o, dtype), _dev(c0))
    df, dv, do, dc0 = ard.glr_bwd(_dev(f, dtype), _dev(v, dtype), _dev(o, dtype), _dev(dh, dtype), ckpt)
    rh, rcT, states = L.glr_fwd(f, v, o, c0)
    rdf, rdv, rdo, rdc0 = L.glr_bwd(f, v, o, states, dh)
    tol = (40 + 10) * 2.0 ** -24 + 1e-6 + (2.0 ** -8 if dtype == "bf16" else 0)
    for what, got, ref in (("h", h, rh), ("dv", dv, rdv), ("do", do, rdo)):
        assert (np.abs(to_host(got) - ref) <= tol * np.abs(ref)).all(), what
    # (c_{t-1} - v of df does cancel: against its terms)
    assert (np.abs(to_host(df) - rdf) <= tol * np.abs(rdv) * L.sigmoid(f) * (states[:T] + v)).all()


def test_a_nan_stays_in_its_channel():
    T, B, H = 300, 2, 70
    f, v, o, dh, c0, dcT = _inputs(T, B, H, "f32", True, 2)
    clean = [_dev(x) for x in (f, v, o, dh)]
    h0, cT0, _ = ard.glr_fwd(*clean[:3], c0=_dev(c0))
    for at in ((0, 5), (1, 6)):   # f, v
        bad = [x.clone() for x in clean]
        bad[at[0]][100, 1, at[1]] = float("nan")
        h, cT, ckpt = ard.glr_fwd(*bad[:3], c0=_dev(c0))
        same = torch.ones_like(h, dtype=torch.bool)
        same[100:, 1, at[1]] = False
        assert torch.equal(h[same], h0[same]) and torch.isnan(h[~same]).all() and torch.isnan(cT[1, at[1]])


def test_a_step_in_place_is_the_long_call():
    """Generation: single steps, the state updated in its place, against one call over all steps."""
    T, B, H = 20, 6, 100
    for dtype in ("f32", "bf16"):
        f, v, o, dh, c0, dcT = _inputs(T, B, H, dtype, True, 3)
        fd, vd, od = (_dev(x, dtype) for x in (f, v, o))
        h, cT, _ = ard.glr_fwd(fd, vd, od, _dev(c0), train=False)
        c = _dev(c0)
        for t in range(T):
            ht, c2, _ = ard.glr_fwd(fd[t:t + 1], vd[t:t + 1], od[t:t + 1], c, train=False, out=(None, c, None))
            assert c2.data_ptr() == c.data_ptr()
            assert_parity(ht, to_host(h[t:t + 1]), dtype, None, "h of a step", rounded_ref=True)
        assert_parity(c, to_host(cT), "f32", None, "state after the steps")
        with pytest.raises(ard.ArdError):   # of many steps every workgroup of a sequence reads the first state
            ard.glr_fwd(fd, vd, od, c, train=False, out=(None, c, None))


def test_same_bits_on_every_call_and_in_a_graph():
    T, B, H = 3000, 1, 200
    f, v, o, dh, c0, dcT = _inputs(T, B, H, "bf16", True, 4)
    fd, vd, od, dhd = (_dev(x, "bf16") for x in (f, v, o, dh))
    c0d, dcTd = _dev(c0), _dev(dcT)
    out = (torch.empty_like(fd), torch.empty_like(c0d), torch.empty((-(-T // ard.GLR_CHUNK), B, H), device="cuda"))
    grads = tuple(torch.empty_like(fd) for _ in range(3)) + (torch.empty_like(c0d),)
    ws = torch.empty(ard.glr_workspace_bytes(ard.BF16, T, B, H), dtype=torch.uint8, device="cuda")

    def step():
        ard.glr_fwd(fd, vd, od, c0d, out=out, ws=ws)
        ard.glr_bwd(fd, vd, od, dhd, out[2], dcTd, out=grads, ws=ws)
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
    T, B, H = 900, 2, 60
    f, v, o, dh, c0, dcT = _inputs(T, B, H, "f32", True, 5)
    fd, vd, od, dhd, c0d, dcTd = (_dev(x) for x in (f, v, o, dh, c0, dcT))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    h, cT, ckpt = ard.glr_fwd(fd, vd, od, c0d, stream=side)
    grads = ard.glr_bwd(fd, vd, od, dhd, ckpt, dcTd, stream=side)
    side.synchronize()
    rh, rcT, states = L.glr_fwd(f, v, o, c0)
    _compare("f32", (rh, rcT) + L.glr_bwd(f, v, o, states, dh, dcT), (h, cT) + grads, None)


def test_steps_beyond_32_bit_offsets():
    """Steps 2^30 elements apart: the last starts 4 GB into its buffer."""
    T, B, H, far = 3, 2, 10, 1 << 30
    f, v, o, dh, c0, dcT = _inputs(T, B, H, "bf16", False, 6)
    Z = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda")
    O = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda")
    fd, vd = (Z[at:].as_strided((T, B, H), (far, H)+(1,)) for at in (0, 32))
    fd.copy_(_dev(f, "bf16")), vd.copy_(_dev(v, "bf16"))
    hO, dfO, dvO = (O[at:].as_strided((T, B, H), (far, H, 1)) for at in (0, 20, 40))
    h, cT, ckpt = ard.glr_fwd(fd, vd, None, _dev(c0), out=(hO, None, None))
    rh, rcT, states = L.glr_fwd(f, v, None, c0)
    grads = ard.glr_bwd(fd, vd, None, _dev(dh, "bf16"), ckpt, _dev(dcT), out=(dfO, dvO, None))
    _compare("bf16", (rh, rcT) + L.glr_bwd(f, v, None, states, dh, dcT), (h, cT) + grads, None)


def test_gradient_against_differences_of_the_forward_pass():
    T, B, H = 60, 2, 30
    f, v, o, dh, c0, dcT = _inputs(T, B, H, "f32", True, 7, spread=2.0)
    fd, vd, od, dhd = (_dev(x) for x in (f, v, o, dh))
    _, _, ckpt = ard.glr_fwd(fd, vd, od, _dev(c0))
    grads = [to_host(t) for t in ard.glr_bwd(fd, vd, od, dhd, ckpt, _dev(dcT))]

    def loss(*x):
        h, cT, _ = L.glr_fwd(*x)
        return float((h * dh).sum() + (cT * dcT).sum())
    rng = np.random.default_rng(8)
    for i, at in enumerate((f, v, o, c0)):
        way, args, e = rng.standard_normal(at.shape), [f, v, o, c0], 1e-5
        args[i] = at + e * way
        up = loss(*args)
        args[i] = at - e * way
        diff, got = (up - loss(*args)) / (2 * e), float((grads[i] * way).sum())
        # (as for the norm: e^2 of the third derivative, 1e-16 / e of rounding, 1e-5 of the kernel's gradient's length)
        assert abs(diff - got) <= 2e-5 * np.linalg.norm(grads[i]) * np.linalg.norm(way) / np.sqrt(way.size) + 1e-6 * abs(diff)


@pytest.mark.parametrize("what,error", [("dtype", TypeError), ("strides", ValueError), ("rank", ValueError), ("lengths", ValueError), ("lengths_dtype", TypeError),
                                        ("state", ValueError), ("H", ValueError), ("overlap", ValueError), ("channels", AssertionError)])
def test_refusals(what, error):
    f, v = (torch.zeros((4, 3, 8), device="cuda") for _ in range(2))
    calls = dict(dtype=lambda: ard.glr_fwd(f.half(), v.half()), strides=lambda: ard.glr_fwd(f, v.transpose(0, 1).contiguous().transpose(0, 1)),
                 rank=lambda: ard.glr_fwd(f[0], v[0]), lengths=lambda: ard.glr_fwd(f, v, lengths=torch.zeros(2, dtype=torch.int32, device="cuda")),
                 lengths_dtype=lambda: ard.glr_fwd(f, v, lengths=torch.zeros(3, dtype=torch.int64, device="cuda")),
                 state=lambda: ard.glr_fwd(f, v, c0=torch.zeros(3, 7, device="cuda")), H=lambda: ard.glr_fwd(f, v, H=9),
                 overlap=lambda: ard.glr_fwd(f, v, out=(torch.zeros((1, 3, 8), device="cuda").expand(4, 3, 8), None, None)),
                 channels=lambda: ard.glr_fwd(torch.zeros((4, 8, 3), device="cuda").transpose(1, 2), v))
    with pytest.raises(error):
        calls[what]()
    torch.cuda.synchronize()
