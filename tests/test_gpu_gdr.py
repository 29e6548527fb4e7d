"""The gated delta rule's kernels against the step-by-step oracle: lengths around the chunks, every size of head, heads that share keys,
sequences of unequal length, gates that let nothing or all through."""
import numpy as np
import pytest
import torch

from oracle import gdr as L
from paper_2203_05705_amd import binding as ard
from util import assert_parity, from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances: util's.  Products of fp32 values are as good as fp32's own (three parts of 8 bits each); sums over 64 steps and up to 128 channels, of
# mixed signs, in chains of at most 12 products of 32 each: some 2^-24 x sqrt(128) of their terms' size, 7e-7; what a chunk passes to the next
# is multiplied by matrices of norm at most 1, so errors of n chunks of memory add up like sqrt(n).  fp32 1e-5 leaves ten times that.
# bf16: one rounding of each result, 2^-9, and factors of results kept to 2^-17.

CODE = dict(f32=ard.F32, bf16=ard.BF16)
NAMES = ("dq", "dk", "dv", "df", "db", "dS0")


def _inputs(T, B, Hk, H, Dk, Dv, dtype, seed, spread=5.0):
    rng = np.random.default_rng(seed)
    q, k = (stored(rng.standard_normal((T, B, Hk, Dk)), dtype) for _ in range(2))
    v, do = (stored(rng.standard_normal((T, B, H, Dv)), dtype) for _ in range(2))
    f = stored(rng.standard_normal((T, B, H)) + spread * rng.random(H), dtype)
    b = stored(rng.standard_normal((T, B, H)), dtype)
    S0, dST = (rng.standard_normal((B, H, Dk, Dv)).astype(np.float32).astype(np.float64) for _ in range(2))
    return [q, k, v, f, b], do, S0, dST


def _lengths(T, B, seed):
    n = np.random.default_rng(seed).integers(0, T + 1, B)
    for i, x in enumerate((0, T, min(1, T), min(64, T), min(65, T))):
        if i < B - 1:
            n[i] = x
    return n.astype(np.int32)


def _dead(n, T, B, shape):
    return None if n is None else np.broadcast_to((np.arange(T)[:, None] >= n[None, :]).reshape((T, B) + (1,) * (len(shape) - 2)), shape)


def _compare(dtype, n, o, ro, grads, rgrads):
    T, B = ro.shape[:2]
    assert_parity(o.contiguous(), ro, dtype, _dead(n, T, B, ro.shape), "o")
    for what, g, r in zip(NAMES, grads, rgrads):
        if what == "dS0":
            assert_parity(g.contiguous(), r, "f32", None, what)
        else:
            assert_parity(g.contiguous(), r, dtype, _dead(n, T, B, r.shape), what)


def _check(T, B, Hk, H, Dk, Dv, dtype="f32", ragged=False, start=True, seed=0, scale=None, spread=5.0, x=None, train=True):
    given, do, S0, dST = _inputs(T, B, Hk, H, Dk, Dv, dtype, seed, spread)
    x = given if x is None else x
    n = _lengths(T, B, seed) if ragged else None
    if not start:
        S0 = dST = None
    s = Dk ** -0.5 if scale is None else scale
    ro, rST, states = L.gdr_fwd(*x, S0, n, s)
    xd, dod = [from_vals(t, dtype) for t in x], from_vals(do, dtype)
    nd = None if n is None else torch.from_numpy(n).cuda()
    if n is not None:   # what lies behind a sequence has no part in anything
        for t in xd + [dod]:
            for i in range(B):
                t[n[i]:, i] = float("nan") if i % 2 else float("inf")
    dev = lambda a: None if a is None else from_vals(a, "f32")  # noqa: E731
    o, ST, ckpt = ard.gdr_fwd(*xd, S0=dev(S0), lengths=nd, scale=scale, train=train)
    assert_parity(ST, rST, "f32", None, "ST")
    if not train:
        assert ckpt is None
        assert_parity(o, ro, dtype, _dead(n, T, B, ro.shape), "o")
        return
    assert ckpt.shape == (-(-T // ard.GDR_CHUNK), B, H, Dk, Dv)
    assert_parity(ckpt, states[0:T:ard.GDR_CHUNK], "f32", None, "states kept")
    grads = ard.gdr_bwd(*xd, dod, ckpt, dST=dev(dST), lengths=nd, scale=scale)
    _compare(dtype, n, o, ro, grads, L.gdr_bwd(*x, states, do, dST, n, s))
    again, ST2, none = ard.gdr_fwd(*xd, S0=dev(S0), lengths=nd, scale=scale, train=False)
    assert none is None and np.array_equal(raw_bits(again), raw_bits(o)) and torch.equal(ST, ST2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 4, 5, 8, 9, 15, 16, 17, 31, 33, 48, 63, 64, 65, 127, 128, 129, 200, 321])
def test_steps_around_the_chunks(T, dtype):
    _check(T, 2, 1, 2, 24, 40, dtype, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(1, 1), (2, 3), (4, 8), (7, 9), (15, 17), (16, 16), (31, 33), (32, 64), (60, 125), (63, 65), (64, 64), (65, 63), (64, 128), (96, 66), (100, 8), (127, 127),
                                   (128, 64), (128, 128)])
def test_sizes_of_heads(Dk, Dv, dtype):
    _check(70, 2, 1, 1, Dk, Dv, dtype, seed=Dk + Dv)
    _check(7, 2, 1, 2, Dk, Dv, dtype, ragged=True, seed=Dk * Dv)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,Hk,H", [(1, 1, 1), (1, 3, 3), (3, 1, 4), (2, 2, 6), (5, 4, 4)])
def test_heads_that_share_keys(B, Hk, H, dtype):
    _check(67, B, Hk, H, 32, 48, dtype, seed=H)
    _check(3, B, Hk, H, 32, 48, dtype, seed=H + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("start", [True, False])
@pytest.mark.parametrize("T,B", [(1, 6), (4, 7), (35, 8), (64, 6), (130, 7), (257, 6)])
def test_sequences_of_unequal_length(T, B, start, dtype):
    _check(T, B, 1, 2, 20, 24, dtype, ragged=True, start=start, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (128, 24), (30, 128)])
def test_many_chunks(Dk, Dv, dtype):
    _check(700, 1, 1, 2, Dk, Dv, dtype, seed=1, spread=8.0)
    _check(700, 3, 2, 2, Dk, Dv, dtype, ragged=True, seed=2)


# Few heads of a long sequence are walked in segments: a state passes their transitions as products, which have the chunks' own digits.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,H,Dk,Dv", [(1024, 1, 1, 64, 64), (1100, 2, 1, 128, 128), (1473, 1, 2, 30, 72), (2049, 1, 1, 96, 10), (1601, 3, 2, 64, 33)])
def test_segments_of_long_sequences(T, B, H, Dk, Dv, dtype):
    _check(T, B, 1, H, Dk, Dv, dtype, seed=T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("start", [True, False])
def test_segments_behind_a_sequences_end(start, dtype):
    _check(1700, 7, 1, 1, 40, 70, dtype, ragged=True, start=start, seed=17)
    _check(2500, 6, 1, 1, 66, 24, dtype, ragged=True, start=start, seed=18, spread=9.0)   # (states that last through segments)


def test_segments_of_states_in_the_place_of_what_they_are_made_from():
    T = 1300
    x, do, S0, dST = _inputs(T, 2, 1, 1, 64, 100, "bf16", 3, 9.0)
    xd, dod, s, d = [from_vals(t, "bf16") for t in x], from_vals(do, "bf16"), from_vals(S0, "f32"), from_vals(dST, "f32")
    o, ST, ck = ard.gdr_fwd(*xd, S0=s)
    *g, dS0 = ard.gdr_bwd(*xd, dod, ck, dST=d)
    o2, same, _ = ard.gdr_fwd(*xd, S0=s, out=(None, s, None))
    assert same is s and torch.equal(s, ST) and np.array_equal(raw_bits(o2), raw_bits(o))
    *g2, same = ard.gdr_bwd(*xd, dod, ck, dST=d, out=(None,) * 5 + (d,))
    assert same is d and torch.equal(d, dS0)
    for a, b in zip(g, g2):
        assert np.array_equal(raw_bits(a), raw_bits(b))


def test_a_nan_passes_segments_in_its_column_alone():
    T = 1500
    x, do, S0, _ = _inputs(T, 1, 1, 1, 32, 40, "f32", 5)
    xd = [from_vals(t, "f32") for t in x]
    clean = ard.gdr_fwd(*xd)
    xd[2][10, 0, 0, 7] = float("nan")
    o, ST, ck = ard.gdr_fwd(*xd)
    others = [c for c in range(40) if c != 7]
    assert bool(torch.isnan(ST[..., 7]).all()) and torch.equal(ST[..., others], clean[1][..., others])
    assert bool(torch.isnan(o[64:, ..., 7]).all()) and torch.equal(o[..., others], clean[0][..., others])


@pytest.mark.parametrize("T", [3, 40, 140])
def test_gates_that_let_nothing_or_all_through(T):
    x, *_ = _inputs(T, 2, 1, 3, 16, 16, "f32", 5)
    rng = np.random.default_rng(6)
    ends = np.array([-np.inf, -1e30, -3e4, -200.0, -90.0, 90.0, 1e30, np.inf])
    for i in (3, 4):
        x[i] = np.where(rng.random(x[i].shape) < 0.5, rng.choice(ends, x[i].shape), x[i])
    _check(T, 2, 1, 3, 16, 16, "f32", seed=5, x=[stored(t, "f32") for t in x])
    for f, b in ((-np.inf, np.inf), (np.inf, np.inf), (np.inf, -np.inf), (-1e4, 0.0)):
        x[3][:], x[4][:] = f, b
        _check(T, 2, 1, 3, 16, 16, "f32", seed=5, x=[stored(t, "f32") for t in x])


def test_keys_that_repeat_and_keys_of_zero():
    """The same key at every step makes A full of ones below its diagonal; a key or query of zeros writes and reads nothing."""
    T, D = 130, 32
    for dtype in ("f32", "bf16"):
        x, *_ = _inputs(T, 2, 1, 2, D, D, dtype, 7)
        x[1][:] = x[1][:1]
        x[3][:], x[4][:] = 20.0, 20.0
        _check(T, 2, 1, 2, D, D, dtype, seed=7, x=x)
        x, *_ = _inputs(T, 2, 1, 2, D, D, dtype, 8)
        x[1][::3], x[0][1::3] = 0.0, 0.0
        o = _inputs(T, 2, 1, 2, D, D, dtype, 8)
        S0, dST = o[2], o[3]
        ro, rST, _ = L.gdr_fwd(*x, S0, None, D ** -0.5)
        got, ST, _ = ard.gdr_fwd(*[from_vals(t, dtype) for t in x], S0=from_vals(S0, "f32"))
        assert_parity(got, ro, dtype, None, "o")
        assert_parity(ST, rST, "f32", None, "ST")


def test_fast_decay_keeps_digits_inside_a_chunk():
    """One step that forgets all between steps that forget nothing: differences of sums near 10^4 count to their last digit."""
    T = 128
    x, *_ = _inputs(T, 1, 1, 1, 32, 32, "f32", 9)
    x[3][:] = 8.0
    x[3][20], x[3][90] = -9e3, -60.0
    _check(T, 1, 1, 1, 32, 32, "f32", seed=9, x=[stored(t, "f32") for t in x])


def test_lengths_of_keys_from_tiny_to_large():
    T = 70
    x, *_ = _inputs(T, 2, 1, 1, 40, 24, "f32", 10)
    size = 10.0 ** np.random.default_rng(11).uniform(-1, 6, (T, 2, 1, 1))
    x[0], x[1] = stored(x[0] * size, "f32"), stored(x[1] * size[::-1], "f32")
    S0, dST, do = (_inputs(T, 2, 1, 1, 40, 24, "f32", 10)[i] for i in (2, 3, 1))
    ro, rST, states = L.gdr_fwd(*x, S0, None, 1.0)
    xd = [from_vals(t, "f32") for t in x]
    o, ST, ckpt = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"), scale=1.0)
    grads = ard.gdr_bwd(*xd, from_vals(do, "f32"), ckpt, dST=from_vals(dST, "f32"), scale=1.0)
    rgrads = L.gdr_bwd(*x, states, do, dST, None, 1.0)
    assert_parity(o, ro, "f32", None, "o")
    for what, g, r, by in zip(NAMES, grads, rgrads, (size, size[::-1], 1, 1, 1, 1)):     # the gradient of a long key is as small as the key is long
        d, ref = to_host(g) * by, r * by
        assert np.max(np.abs(d - ref)) <= 1e-5 * np.max(np.abs(ref)), what


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Dk,Dv", [(1, 24, 40), (67, 24, 40), (67, 64, 64), (3, 33, 31), (130, 33, 31)])
def test_parts_of_one_products_rows(T, Dk, Dv, dtype):
    """Inputs and gradients as parts of rows, at odd offsets, time or batch outermost; what lies between is left alone."""
    B, Hk, H = 3, 2, 4
    x, do, S0, dST = _inputs(T, B, Hk, H, Dk, Dv, dtype, T)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    widths = [Hk * Dk, Hk * Dk, H * Dv, H, H]
    s = Dk ** -0.5
    ro, rST, states = L.gdr_fwd(*x, S0, None, s)
    rgrads = L.gdr_bwd(*x, states, do, dST, None, s)
    for batch_outer in (False, True):
        def parts(extra):
            wide = sum(widths) + extra
            Z = torch.full((B, T, wide) if batch_outer else (T, B, wide), 7.0, dtype=t, device="cuda")
            V = Z.transpose(0, 1) if batch_outer else Z
            at, out = 1, []
            for i, w in enumerate(widths):
                p = V[..., at:at + w]
                out.append(p.unflatten(-1, ((Hk, Dk), (Hk, Dk), (H, Dv))[i]) if i < 3 else p)
                at += w
            return Z, out
        Z, xd = parts(4)
        for p, v in zip(xd, x):
            p.copy_(from_vals(v, dtype))
        O = torch.full((B, T, H * Dv + 3) if batch_outer else (T, B, H * Dv + 3), 7.0, dtype=t, device="cuda")
        o = (O.transpose(0, 1) if batch_outer else O)[..., 2:2 + H * Dv].unflatten(-1, (H, Dv))
        gotten, ST, ckpt = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"), out=(o, None, None))
        assert gotten is o or gotten.data_ptr() == o.data_ptr()
        dZ, dxd = parts(9)
        grads = ard.gdr_bwd(*xd, from_vals(do, dtype), ckpt, dST=from_vals(dST, "f32"), out=(*dxd, None))
        _compare(dtype, None, o, ro, grads, rgrads)
        assert bool((O[..., :2] == 7).all() and (O[..., 2 + H * Dv:] == 7).all() and (dZ[..., :1] == 7).all() and (dZ[..., 1 + sum(widths):] == 7).all())


@pytest.mark.parametrize("T", [1, 3, 40, 150])
def test_states_in_the_place_of_what_they_are_made_from(T):
    x, do, S0, dST = _inputs(T, 3, 1, 2, 40, 24, "bf16", 12)
    xd, dod = [from_vals(t, "bf16") for t in x], from_vals(do, "bf16")
    o, ST, ckpt = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"))
    grads = ard.gdr_bwd(*xd, dod, ckpt, dST=from_vals(dST, "f32"))
    s, d = from_vals(S0, "f32"), from_vals(dST, "f32")
    o2, ST2, _ = ard.gdr_fwd(*xd, S0=s, out=(None, s, None), train=False)
    assert ST2 is s and torch.equal(s, ST) and torch.equal(o, o2)
    got = ard.gdr_bwd(*xd, dod, ckpt, dST=d, out=(None,) * 5 + (d,))
    assert got[5] is d and all(torch.equal(p, q) for p, q in zip(got, grads))


def test_steps_of_generation_are_the_long_call():
    T, B, Hk, H, D = 70, 3, 2, 4, 64
    for dtype in ("f32", "bf16"):
        x, _, S0, _ = _inputs(T, B, Hk, H, D, D, dtype, 13)
        xd = [from_vals(t, dtype) for t in x]
        o, ST, _ = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"), train=False)
        s = from_vals(S0, "f32")
        for t in range(T):
            ot = ard.gdr_fwd(*[p[t:t + 1] for p in xd], S0=s, train=False, out=(None, s, None))[0]
            assert_parity(ot, to_host(o[t:t + 1]), dtype, None, "o of a step", rounded_ref=True)
        assert_parity(s, to_host(ST), "f32", None, "state after the steps")


def test_same_bits_on_every_call_and_in_a_graph():
    T, B, Hk, H, D = 200, 2, 1, 2, 64
    x, do, S0, dST = _inputs(T, B, Hk, H, D, D, "bf16", 14)
    xd, dod, s, d = [from_vals(t, "bf16") for t in x], from_vals(do, "bf16"), from_vals(S0, "f32"), from_vals(dST, "f32")
    n = torch.tensor([T, 77], dtype=torch.int32, device="cuda")
    out = [torch.empty_like(dod), torch.empty_like(s), torch.empty((4, B, H, D, D), device="cuda")]
    grads = [torch.empty_like(t) for t in xd] + [torch.empty_like(s)]
    ws = [torch.empty(ard.gdr_workspace_bytes(ard.BF16, T, B, Hk, H, D, D, back), dtype=torch.uint8, device="cuda") for back in (False, True)]

    def step():
        ard.gdr_fwd(*xd, S0=s, lengths=n, out=out, ws=ws[0])
        ard.gdr_bwd(*xd, dod, out[2], dST=d, lengths=n, out=grads, ws=ws[1])
    step()
    torch.cuda.synchronize()
    want = [raw_bits(t) for t in out + grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in out + grads:
            t.fill_(7)
        for w in ws:
            w.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(raw_bits(t), w) for t, w in zip(out + grads, want))


def test_a_stream_of_its_own():
    x, do, S0, dST = _inputs(100, 2, 1, 2, 32, 32, "f32", 15)
    xd, dod, s, d = [from_vals(t, "f32") for t in x], from_vals(do, "f32"), from_vals(S0, "f32"), from_vals(dST, "f32")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    o, ST, ckpt = ard.gdr_fwd(*xd, S0=s, stream=side)
    grads = ard.gdr_bwd(*xd, dod, ckpt, dST=d, stream=side)
    side.synchronize()
    ro, rST, states = L.gdr_fwd(*x, S0, None, 32 ** -0.5)
    _compare("f32", None, o, ro, grads, L.gdr_bwd(*x, states, do, dST, None, 32 ** -0.5))


@pytest.mark.parametrize("T,far", [(3, 1 << 30), (66, 1 << 25)])
def test_steps_beyond_32_bit_offsets(T, far):
    """Steps so far apart that the last starts 4 GB into its buffer."""
    B, H, Dk, Dv = 1, 1, 10, 12
    x, do, S0, dST = _inputs(T, B, H, H, Dk, Dv, "bf16", 16)
    Z = torch.empty((T - 1) * far + 200, dtype=torch.bfloat16, device="cuda")
    at, xd = 0, []
    for i, t in enumerate(x):
        w = t[0].size
        xd.append(Z[at:].as_strided(t.shape, (far, w) + ((t.shape[3], 1) if i < 3 else (1,))))
        xd[-1].copy_(from_vals(t, "bf16"))
        at += w
    o = Z[at:].as_strided((T, B, H, Dv), (far, Dv, Dv, 1))
    at += Dv
    _, ST, ckpt = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"), out=(o, None, None))
    ro, rST, states = L.gdr_fwd(*x, S0, None, Dk ** -0.5)
    dxd = []
    for i, t in enumerate(x):
        w = t[0].size
        dxd.append(Z[at:].as_strided(t.shape, (far, w) + ((t.shape[3], 1) if i < 3 else (1,))))
        at += w
    dod = Z[at:].as_strided((T, B, H, Dv), (far, Dv, Dv, 1))
    dod.copy_(from_vals(do, "bf16"))
    grads = ard.gdr_bwd(*xd, dod, ckpt, dST=from_vals(dST, "f32"), out=(*dxd, None))
    _compare("bf16", None, o, ro, grads, L.gdr_bwd(*x, states, do, dST, None, Dk ** -0.5))


def test_a_nan_stays_in_its_sequence_and_head():
    T, B, H, D = 150, 2, 2, 32
    x, *_ = _inputs(T, B, H, H, D, D, "f32", 17)
    xd = [from_vals(t, "f32") for t in x]
    o, ST, _ = ard.gdr_fwd(*xd)
    for i in range(5):
        bad = [t.clone() for t in xd]
        bad[i][100, 1, 1] = float("nan")
        o2, ST2, _ = ard.gdr_fwd(*bad)
        assert torch.equal(o2[:, 0], o[:, 0]) and torch.equal(o2[:, 1, 0], o[:, 1, 0]) and bool(torch.isfinite(o2[:64, 1, 1]).all())
        assert i == 0 or bool(torch.isnan(ST2[1, 1]).any())
        assert bool(torch.isnan(o2[100, 1, 1]).any())


def test_gradient_against_differences_of_the_forward_pass():
    T, B, Hk, H, Dk, Dv = 80, 1, 1, 2, 12, 10
    x, do, S0, dST = _inputs(T, B, Hk, H, Dk, Dv, "f32", 18, spread=2.0)
    xd = [from_vals(t, "f32") for t in x]
    _, _, ckpt = ard.gdr_fwd(*xd, S0=from_vals(S0, "f32"), scale=1.0)
    grads = [to_host(t) for t in ard.gdr_bwd(*xd, from_vals(do, "f32"), ckpt, dST=from_vals(dST, "f32"), scale=1.0)]

    def loss(*y):
        o, ST, _ = L.gdr_fwd(*y, None, 1.0)
        return float((o * do).sum() + (ST * dST).sum())
    rng = np.random.default_rng(19)
    for i, at in enumerate((*x, S0)):
        way, args, e = rng.standard_normal(at.shape), [*x, S0], 1e-5
        args[i] = at + e * way
        up = loss(*args)
        args[i] = at - e * way
        diff, got = (up - loss(*args)) / (2 * e), float((grads[i] * way).sum())
        # e^2 of the third derivative, 1e-16 / e of rounding, 1e-5 of the kernel's gradient's length
        assert abs(diff - got) <= 2e-5 * np.linalg.norm(grads[i]) * np.linalg.norm(way) / np.sqrt(way.size) + 1e-6 * abs(diff)
