"""The operators of a recurrent language model's training program that stand between its products, as cases that
can be timed and compared: layer norm, the gated linear recurrence and the AdamW step.

``run`` computes a case through ``paper_2203_05705_amd.binding`` where ``own`` is set and in elementary torch
operations, in 32 bits, where it is not; ``exact`` gives the same outputs from the definitions in 64 bits.
Sizes are those of this repository's layers (64 x 128 positions of 1024 units, the 1500-unit layer of the
paper's language model with its 35 steps of batch 20, its perceptrons, the 4096-wide layers) and, for the
recurrence, sequences up to 32768 steps.
"""
import math

import torch

own = False

LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 100   # of the AdamW cases
NORM_EPS = 1e-5
BLOCK = 256     # elements that share a scale of an 8-bit state


def listed():
    return [
        # one position of 64 sequences: the norm of a generation step, a call of a few microseconds
        dict(name="norm_step_f32", family="norm", train=False, dtype="f32", wdtype="f32", R=64, D=1024),
        # a layer whose sizes are multiples of nothing, forward and backward
        dict(name="norm_ragged_bf16", family="norm", train=True, dtype="bf16", wdtype="bf16", R=1027, D=1501),
        # the positions of a training batch (64 steps of 128 sequences), forward and backward
        dict(name="norm_train_bf16", family="norm", train=True, dtype="bf16", wdtype="f32", R=8192, D=1024),
        # the widest layer of the benchmarks over a large batch, forward and backward
        dict(name="norm_wide_bf16", family="norm", train=True, dtype="bf16", wdtype="f32", R=16384, D=4096),
        # one step of 128 sequences, state in, state out: what generation calls for every token
        dict(name="glr_step_bf16", family="glr", train=False, dtype="bf16", T=1, B=128, H=1024, dp=1, gate=True, ragged=False),
        # the paper's language model (35 steps, batch 20, 1500 units) under a row pattern, sequences of unequal length
        dict(name="glr_ragged_f32", family="glr", train=True, dtype="f32", T=35, B=20, H=1500, dp=3, gate=True, ragged=True),
        # the LSTM benchmark's layer as a linear recurrence: forward and backward of a training step
        dict(name="glr_train_bf16", family="glr", train=True, dtype="bf16", T=64, B=128, H=1024, dp=1, gate=True, ragged=False),
        # a whole document read at once: one sequence, time is the only long axis
        dict(name="glr_long_bf16", family="glr", train=False, dtype="bf16", T=32768, B=1, H=1024, dp=1, gate=True, ragged=False),
        # long sequences in training, without an output gate
        dict(name="glr_long_train_bf16", family="glr", train=True, dtype="bf16", T=8192, B=4, H=1024, dp=1, gate=False, ragged=False),
        # a small perceptron with its biases, 32-bit states and gradients: launches and tails of small tensors
        dict(name="adamw_mlp_f32", family="adamw", bits=32, gdtype="f32", copies=False, shapes="1024x784,1024,64x1024,64,10x64,10"),
        # two recurrent layers of 1500 units, bf16 gradients and forward weights, 8-bit states
        dict(name="adamw_1500_8bit", family="adamw", bits=8, gdtype="bf16", copies=True, shapes="6000x3000,6000,6000x3000,6000,1500,1500"),
        # four 4096-wide layers, the most that one step updates here
        dict(name="adamw_4096_8bit", family="adamw", bits=8, gdtype="bf16", copies=True, shapes="4096x4096,4096,4096x4096,4096,4096x4096,4096,4096x4096,4096"),
    ]


def _size(rng, lo, hi):
    """A size from lo to hi, even over its logarithm; half of them round, as layer widths mostly are."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        m = 64 if n >= 256 else 8 if n >= 16 else 1
        n = max(m, n // m * m)
    return min(max(n, lo), hi)


def draw(rng):
    family = rng.choice(("norm", "norm", "glr", "glr", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if family == "norm":
        c = dict(family=family, train=rng.random() < 0.6, dtype=dtype, wdtype=rng.choice(("f32", dtype)), R=_size(rng, 1, 16384), D=_size(rng, 64, 8192))
        while c["R"] * c["D"] * (4 if dtype == "f32" else 2) > 16384 * 4096 * 2:
            c["R"] = c["R"] * 3 // 4
        return c
    if family == "glr":
        c = dict(family=family, train=rng.random() < 0.6, dtype=dtype, T=_size(rng, 1, 32768), B=_size(rng, 1, 128), H=_size(rng, 64, 2048),
                 dp=rng.choice((1, 1, 1, 2, 3)), gate=rng.random() < 0.7, ragged=rng.random() < 0.4)
        while c["T"] * c["B"] * c["H"] // c["dp"] * (4 if dtype == "f32" else 2) > 8192 * 4 * 1024 * 2:
            k = "B" if c["B"] > 1 and (c["T"] < 256 or rng.random() < 0.5) else "T" if c["T"] > 1 else "H"
            c[k] = max(1, c[k] * 3 // 4)
        return c
    shapes, left = [], 4 * 4096 * 4096
    for _ in range(rng.randint(1, 12)):
        rows, cols = _size(rng, 8, 4096), _size(rng, 1, 4096)
        if rows * cols + rows > left:
            break
        left -= rows * cols + rows
        shapes += ["%dx%d" % (rows, cols), "%d" % rows]
    return dict(family=family, bits=rng.choice((8, 8, 32)), gdtype=dtype, copies=rng.random() < 0.5, shapes=",".join(shapes or ["64x64"]))


# ---- what a program has in hand before the call -------------------------------------------------------

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _pad8(n):
    return -(-n // 8) * 8


def _kept(case):
    """Kept units of a row pattern of period dp, first unit kept, and the width they are stored in."""
    k = -(-case["H"] // case["dp"])
    return k, k if case["dp"] == 1 else _pad8(k)


def _numels(case):
    return [math.prod(int(d) for d in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["family"] == "norm":
        dt, wt, R, D = _dtype(case["dtype"]), _dtype(case["wdtype"]), case["R"], case["D"]
        # a residual stream: rows of unequal scale and offset
        s["X"] = (_normal(gen, R, D) * (0.5 + torch.rand((R, 1), generator=gen, device="cuda")) + 0.3 * _normal(gen, R, 1)).to(dt)
        s["gamma"], s["beta"] = (1 + 0.1 * _normal(gen, D)).to(wt), (0.1 * _normal(gen, D)).to(wt)
        if case["train"]:
            s["dY"] = _normal(gen, R, D).to(dt)
    elif case["family"] == "glr":
        dt, T, B = _dtype(case["dtype"]), case["T"], case["B"]
        kept, wide = _kept(case)
        n = 3 if case["gate"] else 2
        if case["dp"] == 1:     # one product made all gates of a position: the parts of its rows
            Z, dZ = torch.empty((T, B, n * wide), dtype=dt, device="cuda"), torch.empty((T, B, n * wide), dtype=dt, device="cuda")
            z, s["dz"] = [Z[..., i * wide:(i + 1) * wide] for i in range(n)], [dZ[..., i * wide:(i + 1) * wide] for i in range(n)]
        else:                   # a product for each gate left the kept units, in rows padded to 8
            z, s["dz"] = [[torch.zeros((T, B, wide), dtype=dt, device="cuda") for _ in range(n)] for _ in range(2)]
        # forget gates whose memories last from one step to hundreds
        z[0][..., :kept] = (_normal(gen, T, B, kept) + 5 * torch.rand(kept, generator=gen, device="cuda")).to(dt)
        for t in z[1:]:
            t[..., :kept] = _normal(gen, T, B, kept).to(dt)
        s["z"], s["c0"], s["kept"], s["wide"] = z, _normal(gen, B, kept), kept, wide
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
        if case["train"]:
            s["dh"], s["dcT"] = torch.zeros((T, B, wide), dtype=dt, device="cuda"), _normal(gen, B, kept)
            s["dh"][..., :kept] = _normal(gen, T, B, kept).to(dt)
    else:
        # every tensor at a multiple of the block in one buffer of each kind; the buffers are what comes back
        ns = _numels(case)
        at, total = [], 0
        for n in ns:
            at.append(total)
            total += -(-n // BLOCK) * BLOCK

        def views(flat, per=1):
            return [flat[a // per:a // per + -(-n // per)] for a, n in zip(at, ns)]
        live = torch.zeros(total, device="cuda")
        for t in views(live):
            t.fill_(1)
        spread = torch.exp(_normal(gen, total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1)   # blocks of unequal gradients
        s["p"] = 0.02 * _normal(gen, total) * live
        s["g"] = (1e-3 * _normal(gen, total) * spread * live).to(_dtype(case["gdtype"]))
        m, v = 3e-4 * _normal(gen, total) * spread * live, 1e-6 * (0.1 + torch.rand(total, generator=gen, device="cuda")) * spread.square() * live
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _encode_m(m)
            s["v"], s["v_scale"] = _encode_v(v)
            s["m_value"], s["v_value"] = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
            s["scales"] = [views(s["m_scale"], BLOCK), views(s["v_scale"], BLOCK)]
            s["values"] = [views(s["m_value"]), views(s["v_value"])]
        else:
            s["m"], s["v"], s["scales"] = m, v, [None, None]
        s["w"] = s["p"].to(torch.bfloat16) if case["copies"] else None
        s["lists"] = [views(s[k]) for k in ("p", "g", "m", "v")]
        s["copies"] = views(s["w"]) if case["copies"] else None
    return s


# ---- the plain forms ----------------------------------------------------------------------------------

def _plain_norm(s):
    c, X = s["case"], s["X"].float()
    gamma, beta = s["gamma"].float(), s["beta"].float()
    mean = X.mean(1)
    d = X - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + NORM_EPS)
    xh = d * rstd[:, None]
    out = dict(Y=(xh * gamma + beta).to(s["X"].dtype), mean=mean, rstd=rstd)
    if c["train"]:
        dY = s["dY"].float()
        q = dY * gamma
        dX = rstd[:, None] * (q - q.mean(1)[:, None] - xh * (q * xh).mean(1)[:, None])
        out.update(dX=dX.to(s["X"].dtype), dgamma=(dY * xh).sum(0).to(s["gamma"].dtype), dbeta=dY.sum(0).to(s["gamma"].dtype))
    return out


def _scan(a, b):
    """y_t = a_t y_{t-1} + b_t over the first axis, y before it 0, in log2(T) passes over all of it."""
    n = 1
    while n < a.shape[0]:
        b = torch.cat((b[:n], a[n:] * b[:-n] + b[n:]))
        a = torch.cat((a[:n], a[n:] * a[:-n]))
        n *= 2
    return b


def _plain_glr(s):
    c, kept, wide, dt = s["case"], s["kept"], s["wide"], s["z"][0].dtype
    z = [t[..., :kept].float() for t in s["z"]]
    T = c["T"]
    F, I, v = 1 / (1 + torch.exp(-z[0])), 1 / (1 + torch.exp(z[0])), z[1]
    O = 1 / (1 + torch.exp(-z[2])) if c["gate"] else torch.ones_like(F)

    def stored(t):
        return torch.nn.functional.pad(t.to(dt), (0, wide - kept))
    live = None
    b = I * v
    if s["lengths"] is not None:
        live = (torch.arange(T, device="cuda")[:, None] < s["lengths"][None, :])[..., None]
        F, b = torch.where(live, F, 1.0), torch.where(live, b, 0.0)

    def only(t):
        return t if live is None else torch.where(live, t, 0.0)
    states = _scan(F, torch.cat((b[:1] + F[:1] * s["c0"], b[1:])))
    out = dict(h=stored(only(O * states)), cT=states[-1])
    if c["train"]:
        dh = s["dh"][..., :kept].float()
        q = only(O * dh)
        q = torch.cat((q[:-1], q[-1:] + s["dcT"]))
        # dc_t = q_t + F_{t+1} dc_{t+1}: the same scan from the last step to the first
        dc = _scan(torch.cat((F[:1], F[1:].flip(0))), q.flip(0)).flip(0)
        before = torch.cat((s["c0"][None], states[:-1]))
        out.update(df=stored(only(dc * (before - v) * F * I)), dv=stored(only(dc * I)), dc0=F[0] * dc[0])
        if c["gate"]:
            out["do"] = stored(only(dh * states * O * (1 - O)))
    return out


def _encode_m(m):
    """Signed 8-bit codes of the square root's share of the block's largest magnitude, and that magnitude."""
    b = m.view(-1, BLOCK)
    top = b.abs().amax(1)
    inv = torch.where(top >= 2.0 ** -126, torch.ones_like(top) / top, 0.0)
    c = torch.round(torch.sqrt(b.abs() * inv[:, None]) * 127)
    return torch.where(b < 0, -c, c).to(torch.int8).view(-1), top


def _encode_v(v):
    """Unsigned 8-bit codes of the fourth root's share of the block's largest value, and that value; none but 0 becomes 0."""
    b = v.view(-1, BLOCK)
    top = b.amax(1)
    inv = torch.where(top >= 2.0 ** -126, torch.ones_like(top) / top, 0.0)
    c = torch.round(torch.sqrt(torch.sqrt(b * inv[:, None])) * 255)
    return torch.where((b > 0) & (top[:, None] >= 2.0 ** -126), c.clamp_min(1), c).to(torch.uint8).view(-1), top


def _decode_m(codes, top):
    t = codes.view(-1, BLOCK).float() * (1 / 127)
    return (t * t.abs() * top[:, None]).view(-1)


def _decode_v(codes, top):
    t = codes.view(-1, BLOCK).float() * (1 / 255)
    t = t * t
    return (t * t * top[:, None]).view(-1)


def _plain_adamw(s):
    c, p, g = s["case"], s["p"], s["g"].float()
    eight = c["bits"] == 8
    m, v = (_decode_m(s["m"], s["m_scale"]), _decode_v(s["v"], s["v_scale"])) if eight else (s["m"], s["v"])
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS
    p.copy_(p * (1 - LR * DECAY) - (LR / (1 - BETA1 ** STEP)) * m / root)
    out = dict(p=p)
    if eight:
        for k, x, encode, decode in (("m", m, _encode_m, _decode_m), ("v", v, _encode_v, _decode_v)):
            codes, top = encode(x)
            s[k].copy_(codes)
            s[k + "_scale"].copy_(top)
            s[k + "_value"].copy_(decode(codes, top))
            out[k] = s[k + "_value"]
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out.update(m=s["m"], v=s["v"])
    if c["copies"]:
        s["w"].copy_(p)
        out["w"] = s["w"]
    return out


# ---- the framework's operators ------------------------------------------------------------------------

def _own_norm(ard, s):
    Y, mean, rstd = ard.layer_norm_fwd(s["X"], s["gamma"], s["beta"], eps=NORM_EPS)
    out = dict(Y=Y, mean=mean, rstd=rstd)
    if s["case"]["train"]:
        out["dX"], out["dgamma"], out["dbeta"] = ard.layer_norm_bwd(s["dY"], s["X"], s["gamma"], mean, rstd)
    return out


def _own_glr(ard, s):
    c = s["case"]
    f, v, o = (s["z"] + [None])[:3]
    H = None if s["kept"] == s["wide"] else s["kept"]
    h, cT, ckpt = ard.glr_fwd(f, v, o, c0=s["c0"], lengths=s["lengths"], train=c["train"], H=H)
    out = dict(h=h, cT=cT)
    if c["train"]:
        df, dv, do = (s["dz"] + [None])[:3]
        dc0 = ard.glr_bwd(f, v, o, s["dh"], ckpt, dcT=s["dcT"], lengths=s["lengths"], H=H, out=(df, dv, do))[3]
        out.update(df=df, dv=dv, dc0=dc0)
        if c["gate"]:
            out["do"] = do
    return out


def _own_adamw(ard, s):
    params, grads, m, v = s["lists"]
    ard.adamw_step(params, grads, m, v, s["scales"][0], s["scales"][1], s["copies"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                   step=STEP)
    out = dict(p=s["p"], m=s["m"], v=s["v"])
    if s["case"]["bits"] == 8:
        ard.adamw_values(m, v, s["scales"][0], s["scales"][1], out=s["values"])
        out.update(m=s["m_value"], v=s["v_value"])
    if s["w"] is not None:
        out["w"] = s["w"]
    return out


def run(state):
    family = state["case"]["family"]
    if not own:
        return dict(norm=_plain_norm, glr=_plain_glr, adamw=_plain_adamw)[family](state)
    from paper_2203_05705_amd import binding as ard
    return dict(norm=_own_norm, glr=_own_glr, adamw=_own_adamw)[family](ard, state)


def work(case):
    """Each input read once, each output written once."""
    if case["family"] == "norm":
        es, ws, n = 4 if case["dtype"] == "f32" else 2, 4 if case["wdtype"] == "f32" else 2, case["R"] * case["D"]
        return dict(bytes=n * es * (4 if case["train"] else 2) + 8 * case["R"] + case["D"] * ws * (4 if case["train"] else 2), flops=n * (22 if case["train"] else 8))
    if case["family"] == "glr":
        es, (kept, wide) = 4 if case["dtype"] == "f32" else 2, _kept(case)
        gates, n, ends = 3 if case["gate"] else 2, case["T"] * case["B"] * wide, case["B"] * kept * 4
        return dict(bytes=n * es * ((2 * gates + 2) if case["train"] else gates + 1) + ends * (4 if case["train"] else 2), flops=n * (40 if case["train"] else 15))
    n = sum(_numels(case))
    state = 2 * 8 if case["bits"] == 32 else 2 * (2 + 4) + 16 / BLOCK
    return dict(bytes=n * (8 + (4 if case["gdtype"] == "f32" else 2) + state + (2 if case["copies"] else 0)), flops=n * (16 if case["bits"] == 32 else 40))


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def _exact_norm(s, train):
    X, gamma, beta = s["X"].double(), s["gamma"].double(), s["beta"].double()
    var, mean = torch.var_mean(X, dim=1, correction=0)
    rstd = (var + NORM_EPS).pow(-0.5)
    xh = (X - mean.unsqueeze(1)) * rstd.unsqueeze(1)
    out = dict(Y=torch.addcmul(beta, xh, gamma), mean=mean, rstd=rstd)
    if train:
        # dX = J^T (gamma dY) with J = rstd (1 - 1/D - xh xh^T / D)
        dY, D = s["dY"].double(), X.shape[1]
        q = dY * gamma
        out["dX"] = rstd.unsqueeze(1) * (q - q.sum(1, keepdim=True) / D - xh * torch.linalg.vecdot(q, xh).unsqueeze(1) / D)
        out["dgamma"], out["dbeta"] = torch.linalg.vecdot(dY, xh, dim=0), dY.sum(0)
    return out


def _exact_glr(s, case):
    """Step by step, as the recurrence is written."""
    kept, wide, T, B = s["kept"], s["wide"], case["T"], case["B"]
    f, v = (s["z"][i][..., :kept].double() for i in (0, 1))
    F, I = torch.sigmoid(f), torch.sigmoid(-f)
    O = torch.sigmoid(s["z"][2][..., :kept].double()) if case["gate"] else torch.ones_like(F)
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    live = (torch.arange(T, device="cuda").unsqueeze(1) < n).unsqueeze(2).double()
    F = F * live + (1 - live)
    I = I * live
    states = torch.empty((T + 1, B, kept), dtype=torch.float64, device="cuda")
    states[0] = s["c0"]
    add = I * v
    for t in range(T):
        torch.addcmul(add[t], F[t], states[t], out=states[t + 1])
    pad = (0, wide - kept)
    out = dict(h=torch.nn.functional.pad(O * states[1:] * live, pad), cT=states[T])
    if case["train"]:
        dh = s["dh"][..., :kept].double() * live
        q = O * dh
        dc = torch.empty_like(q)
        e = s["dcT"].double()
        for t in range(T - 1, -1, -1):
            torch.add(q[t], e, out=dc[t])
            e = F[t] * dc[t]
        out["dc0"] = e
        out["df"] = torch.nn.functional.pad(dc * (states[:-1] - v) * F * I, pad)
        out["dv"] = torch.nn.functional.pad(dc * I, pad)
        if case["gate"]:
            out["do"] = torch.nn.functional.pad(dh * states[1:] * O * (1 - O), pad)
    return out


def _exact_adamw(s, case):
    p, g = s["p"].double(), s["g"].double()
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        share = m / 127
        m = share.abs() * share * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v / 255) ** 4 * s["v_scale"].double().repeat_interleave(BLOCK)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    out = dict(p=p)
    if case["copies"]:
        out["w"] = p
    if case["bits"] == 8:
        tops = [x.abs().view(-1, BLOCK).amax(1).repeat_interleave(BLOCK) for x in (m, v)]
        code = torch.round(127 * (m.abs() / tops[0].clamp_min(1e-300)) ** 0.5)
        m = torch.sign(m) * (code / 127) ** 2 * tops[0]
        code = torch.maximum(torch.round(255 * (v / tops[1].clamp_min(1e-300)) ** 0.25), (v > 0).double())
        v = (code / 255) ** 4 * tops[1]
    out.update(m=m, v=v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["family"] == "norm":
        return _exact_norm(s, case["train"])
    if case["family"] == "glr":
        return _exact_glr(s, case)
    return _exact_adamw(s, case)
