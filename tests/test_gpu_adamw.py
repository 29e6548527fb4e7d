"""The AdamW kernels against the oracle: tensors of every size class and alignment, states in 32 and in 8 bits."""
import numpy as np
import pytest
import torch

from oracle import adamw as A
from paper_2203_05705_amd import binding as ard
from util import from_vals, raw_bits, stored, to_host

pytestmark = pytest.mark.gpu

# tolerances.  States in 32 bits: three operations of half an ulp each, 3 x 2^-24 of the largest term: 4e-7 of |m| + |g|.  The
# parameter: the step is a root, a reciprocal and four products of at most 1 ulp, 1e-6 of the step's size, and p rounds twice, 2e-7 |p|.
# Codes of 8-bit states and their scales: equal, bit for bit (they are defined by operations in 32 bits).

HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.05)


def _case(n, bits, gdtype, seed, t=7):
    rng = np.random.default_rng(seed)
    f32 = lambda x: x.astype(np.float32)  # noqa: E731
    p, g = f32(0.05 * rng.standard_normal(n)), stored(1e-3 * rng.standard_normal(n) * np.exp(rng.standard_normal(n)), gdtype)
    m, v = f32(3e-4 * rng.standard_normal(n)), f32(1e-6 * rng.random(n))
    if bits == 32:
        return p, g, m, v, None, None
    (mc, mt), (vc, vt) = A.encode_m(m), A.encode_v(v)
    return p, g, mc, vc, mt, vt


def _put(a, shift=0):
    """Device copy whose first element lies `shift` elements into its allocation, between bytes that are to stay."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    buf = torch.full((t.numel() + 2 * shift + 8,), 77, dtype=t.dtype, device="cuda")
    view = buf[shift:shift + t.numel()]
    view.copy_(t.view(-1))
    return view.view(t.shape), buf


def _expect(case, bits, t, scale=1.0):
    """(p, m, v) in 64 bits, and the codes and scales of m and v."""
    p, g, m, v, mt, vt = case
    if bits == 8:
        m, v = A.decode_m(m, mt), A.decode_v(v, vt)
    exact = A.step(p.astype(np.float64), g, m.astype(np.float64), v.astype(np.float64), HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"],
                   HYPER["weight_decay"], t, scale)
    if bits == 32:
        return exact, None
    m2, v2 = A.states_f32(g, m, v, HYPER["beta1"], HYPER["beta2"], scale)
    return exact, (A.encode_m(m2), A.encode_v(v2))


def _check(cases, bits, gdtype, t=7, copies=False, shift=0, scale=None):
    lists = dict(p=[], g=[], m=[], v=[], ms=[], vs=[], w=[])
    bufs = []
    for p, g, m, v, mt, vt in cases:
        for k, a in (("p", p), ("m", m), ("v", v)):
            view, buf = _put(a, shift)
            lists[k].append(view)
            bufs.append((buf, shift, view.numel()))
        gd = from_vals(g, gdtype)
        if shift:
            buf = torch.zeros(gd.numel() + shift, dtype=gd.dtype, device="cuda")
            buf[shift:] = gd
            gd = buf[shift:]
        lists["g"].append(gd)
        if bits == 8:
            for k, a in (("ms", mt), ("vs", vt)):
                view, buf = _put(a)
                lists[k].append(view)
                bufs.append((buf, 0, view.numel()))
        wb = torch.full((p.size + 2 * shift + 8,), 77, dtype=torch.bfloat16, device="cuda")
        lists["w"].append(wb[shift:shift + p.size])
        bufs.append((wb, shift, p.size if copies else 0))
    sd = None if scale is None else torch.tensor([scale], dtype=torch.float32, device="cuda")
    ard.adamw_step(lists["p"], lists["g"], lists["m"], lists["v"], lists["ms"] if bits == 8 else None, lists["vs"] if bits == 8 else None,
                   lists["w"] if copies else None, step=t, grad_scale=sd, **HYPER)
    torch.cuda.synchronize()
    for buf, s, n in bufs:
        rest = torch.cat((buf[:s], buf[s + n:])).float()
        assert (rest == 77).all(), "something beside a tensor was written"
    for i, case in enumerate(cases):
        (p, m, v), codes = _expect(case, bits, t, 1.0 if scale is None else scale)
        got = to_host(lists["p"][i])
        move = np.max(np.abs(p - (1 - HYPER["lr"] * HYPER["weight_decay"]) * case[0]), initial=0)   # the largest step
        assert np.max(np.abs(got - p), initial=0) <= 2e-7 * np.max(np.abs(p), initial=0) + 1e-6 * move
        if bits == 8:
            for k, s, (c, top) in (("m", "ms", codes[0]), ("v", "vs", codes[1])):
                assert np.array_equal(lists[k][i].cpu().numpy(), c), f"codes of {k}"
                assert np.array_equal(raw_bits(lists[s][i]), top.view(np.uint32)), f"scales of {k}"
        else:
            big = np.max(np.abs(case[1]), initial=0) * (1.0 if scale is None else scale)
            assert np.max(np.abs(to_host(lists["m"][i]) - m), initial=0) <= 4e-7 * (np.max(np.abs(m), initial=0) + big)
            assert np.max(np.abs(to_host(lists["v"][i]) - v), initial=0) <= 4e-7 * (np.max(np.abs(v), initial=0) + big * big)
        if copies:
            assert torch.equal(lists["w"][i].float(), lists["p"][i].to(torch.bfloat16).float())
    return lists


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 255, 256, 257, 511, 1023, 1025, 4095, 4096, 4097, 8200, 100003])
def test_tensors_of_any_size(n, gdtype, bits):
    _check([_case(n, bits, gdtype, n)], bits, gdtype, copies=n % 2 == 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_tensors_that_start_anywhere(shift, gdtype, bits):
    _check([_case(n, bits, gdtype, n) for n in (3, 256, 5001)], bits, gdtype, copies=True, shift=shift)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_holds(bits):
    rng = np.random.default_rng(3)
    sizes = [int(n) for n in rng.integers(1, 3000, 130)] + [0, 20000, 0, 1]
    _check([_case(n, bits, "f32", i) for i, n in enumerate(sizes)], bits, "f32")
    assert ard.adamw_step([], [], [], []) is None


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("t", [1, 2, 100000])
def test_first_and_late_steps(t, bits):
    n = 3000
    p, g, *_ = _case(n, 32, "f32", 1)
    if t > 1:
        _check([_case(n, bits, "f32", t)], bits, "f32", t=t)
        return
    state = ard.adamw_state([torch.zeros(n, device="cuda")], bits)
    zero = np.zeros(n, np.float32)
    m, v = (zero, zero) if bits == 32 else (zero.astype(np.int8), zero.astype(np.uint8))
    scales = (None, None) if bits == 32 else tuple(state[k][0].cpu().numpy() for k in ("m_scale", "v_scale"))
    assert all(s is None or (s.size == 12 and not s.any()) for s in scales)
    _check([(p, g, m, v) + scales], bits, "f32", t=1)


@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_smallest_normal_number(bits):
    """Gradients of some 1e-19 and an eps that is smaller still: each step within 1e-6 of the formula on the states in 32 bits."""
    n, eps, t = 4096, 1e-32, 1000
    rng = np.random.default_rng(4)
    v = (10.0 ** rng.uniform(-44, -34, n)).astype(np.float32)
    m = (np.sqrt(v.astype(np.float64)) * rng.uniform(0.1, 1, n)).astype(np.float32)
    g = np.where(np.arange(n) % 2, 0, 1e-20 * rng.standard_normal(n)).astype(np.float32)
    p, gd = torch.zeros(n, device="cuda"), from_vals(g, "f32")
    if bits == 8:
        (mc, mt), (vc, vt) = A.encode_m(m), A.encode_v(v)
        m, v = A.decode_m(mc, mt), A.decode_v(vc, vt)
        state = [[torch.from_numpy(a).cuda()] for a in (mc, vc, mt, vt)]
    else:
        state = [[torch.from_numpy(a).cuda()] for a in (m.copy(), v.copy())] + [None, None]
    ard.adamw_step([p], [gd], *state, lr=1e-3, eps=eps, weight_decay=0.0, step=t)
    m, v = (x.astype(np.float64) for x in A.states_f32(g, m, v, 0.9, 0.999))
    assert np.count_nonzero((v > 0) & (v < 2.0 ** -126)) > n // 10
    want = -1e-3 / (1 - 0.9 ** t) * m / (np.sqrt(v) / np.sqrt(1 - 0.999 ** t) + eps)
    assert (np.abs(to_host(p) - want) <= 1e-6 * np.abs(want)).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_scale_that_the_host_does_not_know(bits):
    for scale in (0.25, 0.0, 3.0):
        _check([_case(n, bits, "bf16", n) for n in (10, 3001)], bits, "bf16", scale=scale)
    for scale in (float("nan"), float("inf"), -float("inf")):   # the step is skipped
        case = _case(3001, bits, "bf16", 1)
        p, m, v = (torch.from_numpy(case[i]).cuda() for i in (0, 2, 3))
        scales = [None if s is None else [torch.from_numpy(s).cuda()] for s in case[4:]]
        w = torch.full((3001,), 5.0, dtype=torch.bfloat16, device="cuda")
        before = [t.clone() for t in (p, m, v, w)] + [s[0].clone() for s in scales if s]
        ard.adamw_step([p], [from_vals(case[1], "bf16")], [m], [v], *scales, [w], grad_scale=torch.tensor([scale], device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip([p, m, v, w] + [s[0] for s in scales if s], before))


def test_blocks_without_a_gradient_and_without_numbers():
    """8-bit states: a block of zeros stays one; a NaN or an infinity takes its own block with it and no other; a v above zero stays
    above zero beside a v that is ten orders larger."""
    n = 256 * 5 + 100
    p, g, m, v, mt, vt = _case(n, 8, "f32", 2)
    m[:], v[:], mt[:], vt[:] = 0, 0, 0, 0
    g = g.astype(np.float32)
    g[256:512] = 0
    g[600], g[256 * 4 + 3] = np.nan, np.inf
    g[768:1024] = 1e-6
    g[800] = 1.0
    t = [torch.from_numpy(x).cuda() for x in (p, g, m, v, mt, vt)]
    ard.adamw_step(*[[x] for x in t], **HYPER)
    dm, dv = (x[0].cpu().numpy() for x in ard.adamw_values(*[[x] for x in t[2:]]))
    assert not dm[256:512].any() and not dv[256:512].any()
    for block in (2, 4):
        assert np.isnan(dm[block * 256:(block + 1) * 256]).all() and np.isnan(dv[block * 256:(block + 1) * 256]).all()
    fine = [i for i in range(n) if i // 256 not in (2, 4)]
    assert np.isfinite(dm[fine]).all() and np.isfinite(dv[fine]).all() and np.isfinite(t[0].cpu().numpy()[fine]).all()
    assert (dv[768:1024] > 0).all()
    m2, v2 = A.states_f32(g, np.zeros(n), np.zeros(n), 0.9, 0.999)
    for codes, top, (c, s) in ((t[2], t[4], A.encode_m(m2)), (t[3], t[5], A.encode_v(v2))):
        assert np.array_equal(codes.cpu().numpy()[fine], c[fine]) and np.array_equal(top.cpu().numpy()[[0, 1, 3, 5]], s[[0, 1, 3, 5]])


def test_values_of_every_code():
    m = np.concatenate([np.arange(-127, 128), [-128]]).astype(np.int8)
    v = np.arange(256).astype(np.uint8)
    for top in (1.0, 3.7e-5, 2.0 ** -120, 3e38):
        tops = np.array([top], np.float32)
        args = [[torch.from_numpy(x).cuda()] for x in (m, v, tops, tops)]
        dm, dv = (x[0].cpu().numpy() for x in ard.adamw_values(*args))
        assert np.array_equal(dm, A.decode_m(m, tops)) and np.array_equal(dv, A.decode_v(v, tops))
    out = ([torch.empty(256, device="cuda")], [torch.empty(256, device="cuda")])
    assert ard.adamw_values(*args, out=out) is out and np.array_equal(out[0][0].cpu().numpy(), dm)


def test_values_of_more_tensors_than_a_launch_holds():
    sizes = [1, 255, 257, 5000] * 30 + [0]
    cases = [_case(n, 8, "f32", i) for i, n in enumerate(sizes)]
    args = [[torch.from_numpy(c[k]).cuda() for c in cases] for k in (2, 3, 4, 5)]
    dm, dv = ard.adamw_values(*args)
    for i, c in enumerate(cases):
        assert np.array_equal(dm[i].cpu().numpy(), A.decode_m(c[2], c[4])) and np.array_equal(dv[i].cpu().numpy(), A.decode_v(c[3], c[5]))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_steps_follow_the_formula(bits):
    """Twenty steps on changing gradients: with 32-bit states beside the formula in 64 bits; with 8-bit states codes that equal the
    oracle's at every step."""
    n = 2000
    rng = np.random.default_rng(5)
    p = (0.1 * rng.standard_normal(n)).astype(np.float32)
    pd = torch.from_numpy(p.copy()).cuda()
    st = ard.adamw_state([pd], bits)
    ref = (p.astype(np.float64), np.zeros(n), np.zeros(n))
    for t in range(1, 21):
        g = (1e-2 * rng.standard_normal(n)).astype(np.float32)
        ard.adamw_step([pd], [torch.from_numpy(g).cuda()], st["m"], st["v"], st["m_scale"], st["v_scale"], step=t, **HYPER)
        if bits == 8:
            m2, v2 = A.states_f32(g, ref[1], ref[2], HYPER["beta1"], HYPER["beta2"])
            mc, vc = A.encode_m(m2), A.encode_v(v2)
            assert np.array_equal(st["m"][0].cpu().numpy(), mc[0]) and np.array_equal(st["v"][0].cpu().numpy(), vc[0])
        ref = A.step(*[ref[0], g.astype(np.float64)] + list(ref[1:]), *HYPER.values(), t)
        if bits == 8:
            ref = (ref[0], A.decode_m(*mc), A.decode_v(*vc))
    assert np.max(np.abs(to_host(pd) - ref[0])) <= 20 * (2e-7 * np.max(np.abs(ref[0])) + 1e-6 * HYPER["lr"] * 10)


def test_a_graph_and_a_stream():
    case = _case(9000, 8, "bf16", 6)
    g = from_vals(case[1], "bf16")

    def fresh():
        return [torch.from_numpy(case[i].copy()).cuda() for i in (0, 2, 3, 4, 5)]
    want = fresh()
    for _ in range(3):
        ard.adamw_step([want[0]], [g], *[[x] for x in want[1:]], step=3, **HYPER)
    got, other = fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ard.adamw_step([got[0]], [g], *[[x] for x in got[1:]], step=3, **HYPER)
    side = torch.cuda.Stream()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ard.adamw_step([other[0]], [g], *[[x] for x in other[1:]], step=3, stream=side, **HYPER)
        side.synchronize()
    for a, b, c in zip(want, got, other):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_elements_than_32_bits_count(bits):
    """A tensor of 2^31 + 513 elements: its first and last thousand against the same elements on their own."""
    n, part = (1 << 31) + 513, 256 * 4 + 1
    small = _case(part, bits, "bf16", 7)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    st = ard.adamw_state([p], bits)
    first = (n - part) // 256 * 256      # a block's start
    at = [slice(0, part - 1), slice(first, n)]
    tail = n - first
    case = _case(tail, bits, "bf16", 8)
    for s, c, k in ((at[0], small, part - 1), (at[1], case, tail)):
        p[s], g[s] = torch.from_numpy(c[0][:k]).cuda(), from_vals(c[1][:k], "bf16")
        st["m"][0][s], st["v"][0][s] = torch.from_numpy(c[2][:k]).cuda(), torch.from_numpy(c[3][:k]).cuda()
        if bits == 8:
            b = slice(s.start // 256, s.start // 256 + -(-k // 256))
            st["m_scale"][0][b], st["v_scale"][0][b] = (torch.from_numpy(x[:-(-k // 256)]).cuda() for x in c[4:])
    ard.adamw_step([p], [g], st["m"], st["v"], st["m_scale"], st["v_scale"], step=7, **HYPER)
    for s, c, k in ((at[0], small, part - 1), (at[1], case, tail)):
        alone = [torch.from_numpy(x[:k].copy()).cuda() for x in (c[0], c[2], c[3])]
        scales = [None, None] if bits == 32 else [[torch.from_numpy(x[:-(-k // 256)].copy()).cuda()] for x in c[4:]]
        ard.adamw_step([alone[0]], [from_vals(c[1][:k], "bf16")], [alone[1]], [alone[2]], *scales, step=7, **HYPER)
        for got, want in zip((p, st["m"][0], st["v"][0]), alone):
            assert torch.equal(got[s], want)
    assert not p[1 << 30:(1 << 30) + 4096].any()


@pytest.mark.parametrize("what,error", [("lists", ValueError), ("dtype", TypeError), ("size", ValueError), ("scales", ValueError), ("one_scale", ValueError),
                                        ("codes", TypeError), ("step", ard.ArdError), ("beta", ard.ArdError), ("eps", ard.ArdError), ("lr", ard.ArdError)])
def test_refusals(what, error):
    p, g, m, v = (torch.zeros(300, device="cuda") for _ in range(4))
    s = [torch.zeros(2, device="cuda")]
    codes = [p.to(torch.int8)], [p.to(torch.uint8)]
    calls = dict(lists=lambda: ard.adamw_step([p], [g, g], [m], [v]), dtype=lambda: ard.adamw_step([p.double()], [g], [m], [v]),
                 size=lambda: ard.adamw_step([p], [g[:299]], [m], [v]), scales=lambda: ard.adamw_step([p], [g], *codes, [s[0][:1]], s),
                 one_scale=lambda: ard.adamw_step([p], [g], *codes, s), codes=lambda: ard.adamw_step([p], [g], [m], [v], s, s),
                 step=lambda: ard.adamw_step([p], [g], [m], [v], step=0), beta=lambda: ard.adamw_step([p], [g], [m], [v], beta1=1.0),
                 eps=lambda: ard.adamw_step([p], [g], [m], [v], eps=0.0), lr=lambda: ard.adamw_step([p], [g], [m], [v], lr=float("nan")))
    with pytest.raises(error):
        calls[what]()
    torch.cuda.synchronize()
    assert not p.any()
    with pytest.raises(ValueError):
        ard.adamw_state([p], 16)
