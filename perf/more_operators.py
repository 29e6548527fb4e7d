"""The operators at the two ends of a recurrent language model and a recurrence with a matrix for a state, as cases that
can be timed and compared: the embedding of tokens, the gated delta rule, and the loss against a teacher's top logits.

``run`` computes a case through ``paper_2203_05705_amd.binding`` where ``own`` is set and in elementary torch
operations, in 32 bits (64 for sums of decays and the inverse inside a chunk), where it is not; ``exact`` gives the same
outputs from the definitions in 64 bits.  Sizes are those of this repository's layers (64 x 128 positions of 1024 units, the
1500-unit language model with its 35 steps of batch 20) with vocabularies from 10000 entries on, and, for the recurrence,
sequences up to 16384 steps.
"""
import math

import torch

own = False

EPS = 1e-6      # beside the squared lengths of keys and queries
CHUNK = 64      # steps that the plain form of the delta rule takes together


def listed():
    return [
        # the tokens of one generation step of 64 sequences, bf16 table: a call of a few microseconds
        dict(name="embed_step_bf16", family="embed", train=False, dtype="bf16", wdtype="bf16", R=64, V=10000, D=1024, add=False),
        # the 1500-unit language model's batch (35 steps of 20), its table in fp32: odd counts of everything but the width
        dict(name="embed_small_f32", family="embed", train=True, dtype="f32", wdtype="f32", R=700, V=10000, D=1500, add=False),
        # the positions of a training batch (64 steps of 128 sequences), fp32 masters, bf16 activations
        dict(name="embed_train_bf16", family="embed", train=True, dtype="bf16", wdtype="f32", R=8192, V=32768, D=1024, add=False),
        # a large batch whose table is the output product's too: its gradient joins the one that is there
        dict(name="embed_large_bf16", family="embed", train=True, dtype="bf16", wdtype="f32", R=131072, V=50000, D=1024, add=True),
        # one step of 128 sequences, states in, states out: what generation calls for every token
        dict(name="gdr_step_bf16", family="gdr", train=False, dtype="bf16", T=1, B=128, Hk=8, H=8, Dk=128, Dv=128, ragged=False),
        # 35 steps of batch 20 in fp32, 1500 value channels in 12 heads, pairs of heads sharing keys, unequal lengths
        dict(name="gdr_ragged_f32", family="gdr", train=True, dtype="f32", T=35, B=20, Hk=6, H=12, Dk=60, Dv=125, ragged=True),
        # 8192 positions of 1024 channels, forward and backward of a training step
        dict(name="gdr_train_bf16", family="gdr", train=True, dtype="bf16", T=1024, B=8, Hk=8, H=8, Dk=128, Dv=128, ragged=False),
        # a whole document read at once: one sequence, time is the only long axis
        dict(name="gdr_long_bf16", family="gdr", train=False, dtype="bf16", T=16384, B=1, Hk=8, H=8, Dk=128, Dv=128, ragged=False),
        # longer sequences in training, narrow heads in pairs that share keys and queries
        dict(name="gdr_narrow_train_bf16", family="gdr", train=True, dtype="bf16", T=4096, B=4, Hk=8, H=16, Dk=64, Dv=64, ragged=False),
        # the loss of the 1500-unit language model's batch against 8 logits a position, fp32, loss alone (validation)
        dict(name="distill_eval_f32", family="distill", train=False, dtype="f32", tdtype="f32", R=700, V=10000, K=8, T=1.0, alpha=1.0, ragged=False),
        # the same with labels and gradient, at a temperature, positions without a label among them
        dict(name="distill_small_f32", family="distill", train=True, dtype="f32", tdtype="f32", R=700, V=10000, K=20, T=2.0, alpha=0.5, ragged=True),
        # a training batch over a large vocabulary, 64 teacher logits a position
        dict(name="distill_train_bf16", family="distill", train=True, dtype="bf16", tdtype="bf16", R=8192, V=32768, K=64, T=2.0, alpha=0.7, ragged=True),
    ]


def _size(rng, lo, hi):
    """A size from lo to hi, even over its logarithm; half of them round, as layer widths mostly are."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        m = 64 if n >= 256 else 8 if n >= 16 else 1
        n = max(m, n // m * m)
    return min(max(n, lo), hi)


def draw(rng):
    family = rng.choice(("embed", "gdr", "gdr", "distill"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    train = rng.random() < 0.65
    if family == "embed":
        c = dict(family=family, train=train, dtype=dtype, wdtype=rng.choice(("f32", dtype)), R=_size(rng, 1, 131072), V=_size(rng, 256, 65536),
                 D=_size(rng, 32, 4096), add=rng.random() < 0.4)
        while (c["R"] * (4 if dtype == "f32" else 2) + c["V"] * 4) * c["D"] > 131072 * 1024 * 2 + 50000 * 1024 * 4:
            k = "R" if c["R"] > c["V"] else "V"
            c[k] = c[k] * 3 // 4
        return c
    if family == "gdr":
        Hk, Dk = rng.randint(1, 8), rng.choice((16, 32, 64, 64, 96, 128, 128, rng.randint(8, 128)))
        c = dict(family=family, train=train, dtype=dtype, T=_size(rng, 1, 16384), B=_size(rng, 1, 128), Hk=Hk, H=Hk * rng.choice((1, 1, 2, 3)), Dk=Dk,
                 Dv=rng.choice((Dk, Dk, rng.randint(8, 128))), ragged=rng.random() < 0.4)
        while c["T"] * c["B"] * c["H"] > 131072 // (4 if dtype == "f32" else 1):
            k = "B" if c["B"] > 1 and (c["T"] < 256 or rng.random() < 0.5) else "T"
            c[k] = max(1, c[k] * 3 // 4)
        return c
    c = dict(family=family, train=train, dtype=dtype, tdtype=rng.choice(("f32", dtype)), R=_size(rng, 1, 8192), V=_size(rng, 256, 131072), K=_size(rng, 1, 128),
             T=rng.choice((1.0, 2.0, 4.0, 1.5)), alpha=rng.choice((1.0, 0.9, 0.5)), ragged=rng.random() < 0.6)
    while c["R"] * c["V"] * (4 if dtype == "f32" else 2) > 8192 * 32768 * 2:
        c["R"] = max(1, c["R"] * 3 // 4)
    return c


# ---- what a program has in hand before the call -------------------------------------------------------

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _shares(V, device="cuda"):
    """How often the words of a language come: the r-th most frequent as 1 / (r + 2.7)."""
    w = 1 / (torch.arange(1, V + 1, dtype=torch.float64, device=device) + 2.7)
    return w / w.sum()


def _sections(case):
    """Widths of q, k, v, f and b in a row of the product that makes them all."""
    return case["Hk"] * case["Dk"], case["Hk"] * case["Dk"], case["H"] * case["Dv"], case["H"], case["H"]


def _parts(case, Z):
    q, k, v, f, b = Z.split(_sections(case), dim=-1)
    return q.unflatten(-1, (case["Hk"], -1)), k.unflatten(-1, (case["Hk"], -1)), v.unflatten(-1, (case["H"], -1)), f, b


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["family"] == "embed":
        dt, wt, R, V, D = _dtype(case["dtype"]), _dtype(case["wdtype"]), case["R"], case["V"], case["D"]
        ranks = torch.searchsorted(_shares(V).cumsum(0), torch.rand(R, generator=gen, device="cuda", dtype=torch.float64)).clamp_max(V - 1)
        ids = torch.randperm(V, generator=gen, device="cuda")[ranks].int()      # tokens are not numbered by frequency
        s["ids"] = torch.where(torch.rand(R, generator=gen, device="cuda") < 0.03, -1, ids)     # positions behind short sequences
        s["E"], s["scale"] = (0.02 * _normal(gen, V, D)).to(wt), math.sqrt(D)
        if case["train"]:
            s["dY"] = (1e-2 * _normal(gen, R, D)).to(dt)
            s["dE"] = 1e-2 * _normal(gen, V, D) if case["add"] else torch.empty((V, D), device="cuda")
    elif case["family"] == "gdr":
        dt, T, B, H, Dk, Dv = _dtype(case["dtype"]), case["T"], case["B"], case["H"], case["Dk"], case["Dv"]
        wide = sum(_sections(case))
        Z = _normal(gen, T, B, wide)
        Z[..., wide - 2 * H:wide - H] += 1 + 5 * torch.rand(H, generator=gen, device="cuda")     # heads forget within a few steps or hundreds
        s["parts"] = _parts(case, Z.to(dt))
        s["S0"] = 0.1 * _normal(gen, B, H, Dk, Dv)
        s["scale"] = Dk ** -0.5
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
        if case["train"]:
            s["do"], s["dST"] = _normal(gen, T, B, H, Dv).to(dt), 0.1 * _normal(gen, B, H, Dk, Dv)
            s["grads"] = _parts(case, torch.zeros((T, B, wide), dtype=dt, device="cuda"))
    else:
        dt, R, V, K = _dtype(case["dtype"]), case["R"], case["V"], case["K"]
        Z = 2 * _normal(gen, R, V)
        teacher = (0.7 * Z + 1.4 * _normal(gen, R, V)).topk(K, dim=1)
        s["Z"], s["t"], s["ids"] = Z.to(dt), teacher.values.to(_dtype(case["tdtype"])).contiguous(), teacher.indices.int().contiguous()
        s["labels"] = None
        if case["alpha"] < 1:
            pick = torch.randint(0, K, (R, 1), generator=gen, device="cuda")
            s["labels"] = s["ids"].gather(1, pick).squeeze(1)
            if case["ragged"]:
                s["labels"] = torch.where(torch.rand(R, generator=gen, device="cuda") < 0.1, -1, s["labels"])
        if case["train"]:
            s["dloss"] = torch.full((R,), 1 / R, device="cuda") * torch.randint(1, 3, (R,), generator=gen, device="cuda")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------

def _plain_embed(s):
    c, dt = s["case"], _dtype(s["case"]["dtype"])
    there = s["ids"] >= 0
    at = s["ids"].long().clamp_min(0)
    out = dict(Y=torch.where(there[:, None], s["scale"] * s["E"][at].float(), 0.0).to(dt))
    if c["train"]:
        if not c["add"]:
            s["dE"].zero_()
        s["dE"].index_add_(0, at, torch.where(there[:, None], s["scale"] * s["dY"].float(), 0.0))
        out["dE"] = s["dE"]
    return out


def _scan(a, b):
    """y_n = a_n y_{n-1} + b_n over the second axis (matrices a, y before it 0), in log2(N) passes over all of it."""
    n = 1
    while n < a.shape[1]:
        b = torch.cat((b[:, :n], a[:, n:] @ b[:, :-n] + b[:, n:]), 1)
        a = torch.cat((a[:, :n], a[:, n:] @ a[:, :-n]), 1)
        n *= 2
    return b


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A, in 64 bits: the product of I + (-A)^(2^i)."""
    P = -A.double()
    M = torch.eye(A.shape[-1], dtype=torch.float64, device=A.device) + P
    n = 2
    while n < A.shape[-1]:
        P = P @ P
        M = M + M @ P
        n *= 2
    return M.float()


def _t(x):
    return x.transpose(-1, -2).contiguous()


def _plain_gdr(s):
    c, dt = s["case"], s["parts"][0].dtype
    T, B, Hk, H, Dk, Dv = (c[k] for k in ("T", "B", "Hk", "H", "Dk", "Dv"))
    q, k, v, f, b = (t.float() for t in s["parts"])
    live = None if s["lengths"] is None else torch.arange(T, device="cuda")[:, None] < s["lengths"][None, :]

    def only(t):
        return t if live is None else torch.where(live.view(T, B, *(1,) * (t.dim() - 2)), t, 0.0)
    N = -(-T // CHUNK)

    def chunks(t):      # [T, B, H, D] -> [B * H, N, CHUNK, D], zeros behind the last step
        t = torch.nn.functional.pad(t, (0,) * (2 * t.dim() - 1) + (N * CHUNK - T,))
        return t.view(N, CHUNK, B, H, -1).permute(2, 3, 0, 1, 4).reshape(B * H, N, CHUNK, -1)

    def steps(t):       # and back
        return t.view(B, H, N, CHUNK, -1).permute(2, 3, 0, 1, 4).reshape(N * CHUNK, B, H, -1)[:T]
    rq, rk = (1 / torch.sqrt((t * t).sum(-1, keepdim=True) + EPS) for t in (q, k))
    qh, kh = q * rq, k * rk
    decay = only(-(torch.log1p(torch.exp(-f.abs())) + (-f).clamp_min(0)))
    w = 1 / (1 + torch.exp(-b))
    Q, K, V, W = chunks(s["scale"] * only(qh).repeat_interleave(H // Hk, 2)), chunks(only(kh).repeat_interleave(H // Hk, 2)), chunks(only(v)), chunks(only(w)[..., None])
    G = chunks(decay[..., None]).double().cumsum(2)
    order = torch.arange(CHUNK, device="cuda")
    upto = order[:, None] >= order[None, :]
    fade = torch.exp(torch.where(upto, G - G.squeeze(3).unsqueeze(2), -torch.inf)).float()
    since, still = torch.exp(G).float(), torch.exp(G[:, :, -1:] - G).float()
    whole = since[:, :, -1:]
    KT = _t(K)
    strictly = (order[:, None] > order[None, :]).float()
    A, P = W * fade * (K @ KT) * strictly, fade * (Q @ KT)
    M = _inverse(A)
    U, R, Kd, Qd = M @ (W * V), M @ (W * since * K), K * still, Q * since
    KdT = _t(Kd)
    turn, add = whole * torch.eye(Dk, device="cuda") - KdT @ R, KdT @ U
    S0 = s["S0"].view(B * H, 1, Dk, Dv)
    states = _scan(turn, torch.cat((add[:, :1] + turn[:, :1] @ S0, add[:, 1:]), 1))
    S = torch.cat((S0, states[:, :-1]), 1)
    U = U - R @ S
    out = dict(o=only(steps(Qd @ S + P @ U)).to(dt), ST=states[:, -1].reshape(B, H, Dk, Dv))
    if not c["train"]:
        return out
    dO = chunks(only(s["do"].float()))
    back, dS = _t(turn), _t(Qd) @ dO - _t(R) @ (_t(P) @ dO)
    last = s["dST"].view(B * H, 1, Dk, Dv)
    ends = _scan(back.flip(1), torch.cat((dS[:, -1:] + back[:, -1:] @ last, dS[:, :-1].flip(1)), 1))
    ends = ends.flip(1)     # gradient of the state before every chunk
    dE = torch.cat((ends[:, 1:], last), 1)      # and behind it
    dX = _t(M) @ (_t(P) @ dO + Kd @ dE)
    UT, ST = _t(U), _t(S)
    dA, dP = -(dX @ UT), dO @ UT
    nA, nP = dA * W * fade * strictly, dP * fade
    dQ_S, dK_S, dK_E = since * (dO @ ST), -W * since * (dX @ ST), still * (U @ _t(dE))
    dQ = dQ_S + nP @ K
    dK = nA @ K + _t(nA) @ K + _t(nP) @ Q + dK_S + dK_E
    into = (dK_E * K).sum(-1, keepdim=True).double()
    pairs = (dA * A + dP * P).double()
    dG = (dQ_S * Q).sum(-1, keepdim=True).double() + (dK_S * K).sum(-1, keepdim=True).double() - into + pairs.sum(3, keepdim=True) - _t(pairs).sum(3, keepdim=True)
    dG[:, :, -1:] += into.sum(2, keepdim=True) + (whole.double() * (S * dE).sum((2, 3), keepdim=True))
    dg = dG.flip(2).cumsum(2).flip(2).float()
    dw = (dX * U).sum(-1, keepdim=True)

    def unit(t, h, r):      # through the division by the length, after the heads that share it are added up
        t = only(steps(t).view(T, B, Hk, H // Hk, Dk).sum(3))
        return (r * (t - h * (h * t).sum(-1, keepdim=True))).to(dt)
    found = unit(dQ * s["scale"], qh, rq), unit(dK, kh, rk), only(steps(W * dX)).to(dt), only(steps(dg).squeeze(3) / (1 + torch.exp(f))).to(dt), \
        only(steps(dw).squeeze(3) * (1 - w)).to(dt)
    return dict(out, dq=found[0], dk=found[1], dv=found[2], df=found[3], db=found[4], dS0=ends[:, 0].reshape(B, H, Dk, Dv))


def _plain_distill(s):
    c, Z, dt = s["case"], s["Z"].float(), s["Z"].dtype
    T, alpha, at = c["T"], c["alpha"], s["ids"].long()

    def softmax(x):
        e = torch.exp(x - x.amax(1, keepdim=True))
        total = e.sum(1, keepdim=True)
        return e / total, (x.amax(1, keepdim=True) + torch.log(total)).squeeze(1)
    t = s["t"].float() / T
    p, t_lse = softmax(t)
    cool, lse = softmax(Z / T)
    loss = alpha * T * T * (p * ((t - t_lse[:, None]) - (Z.gather(1, at) / T - lse[:, None]))).sum(1)
    hard = None
    if s["labels"] is not None:
        hard, hard_lse = softmax(Z)
        there, y = s["labels"] >= 0, s["labels"].long().clamp_min(0)[:, None]
        loss = loss + (1 - alpha) * torch.where(there, hard_lse - Z.gather(1, y).squeeze(1), 0.0)
    out = dict(loss=loss)
    if c["train"]:
        dZ = alpha * T * cool.scatter_add(1, at, -p)
        if hard is not None:
            dZ += (1 - alpha) * there[:, None] * hard.scatter_add(1, y, torch.full_like(y, -1, dtype=torch.float32))
        out["dZ"] = (s["dloss"][:, None] * dZ).to(dt)
    return out


# ---- the framework's operators ------------------------------------------------------------------------

def _own_embed(ard, s):
    c = s["case"]
    out = dict(Y=ard.embed_fwd(s["ids"], s["E"], scale=s["scale"], dtype=_dtype(c["dtype"])))
    if c["train"]:
        out["dE"] = ard.embed_bwd(s["ids"], s["dY"], c["V"], scale=s["scale"], beta=1.0 if c["add"] else 0.0, out=s["dE"])
    return out


def _own_gdr(ard, s):
    c = s["case"]
    o, ST, ckpt = ard.gdr_fwd(*s["parts"], S0=s["S0"], lengths=s["lengths"], scale=s["scale"], eps=EPS, train=c["train"])
    out = dict(o=o, ST=ST)
    if c["train"]:
        dq, dk, dv, df, db, dS0 = ard.gdr_bwd(*s["parts"], s["do"], ckpt, dST=s["dST"], lengths=s["lengths"], scale=s["scale"], eps=EPS, out=(*s["grads"], None))
        out.update(dq=dq, dk=dk, dv=dv, df=df, db=db, dS0=dS0)
    return out


def _own_distill(ard, s):
    c = s["case"]
    loss, _, dZ = ard.distill_fwd(s["Z"], s["ids"], s["t"], labels=s["labels"], temperature=c["T"], alpha=c["alpha"], dloss=s["dloss"] if c["train"] else None)
    return dict(loss=loss, dZ=dZ) if c["train"] else dict(loss=loss)


def run(state):
    family = state["case"]["family"]
    if not own:
        return dict(embed=_plain_embed, gdr=_plain_gdr, distill=_plain_distill)[family](state)
    from paper_2203_05705_amd import binding as ard
    return dict(embed=_own_embed, gdr=_own_gdr, distill=_own_distill)[family](ard, state)


def work(case):
    """Each input read once, each output written once."""
    if case["family"] == "embed":
        es, ws, R, V, D = 4 if case["dtype"] == "f32" else 2, 4 if case["wdtype"] == "f32" else 2, case["R"], case["V"], case["D"]
        found = float((1 - (1 - _shares(V, "cpu")) ** (0.97 * R)).sum())     # rows of the table that are met
        n = R * (4 + D * es) + found * D * ws
        if case["train"]:
            n += R * D * es + (found * 8 if case["add"] else V * 4) * D
        return dict(bytes=int(n), flops=R * D * (2 if case["train"] else 1))
    if case["family"] == "gdr":
        es, n, Dk, Dv, H = 4 if case["dtype"] == "f32" else 2, case["T"] * case["B"], case["Dk"], case["Dv"], case["H"]
        wide, ends = sum(_sections(case)), case["B"] * H * Dk * Dv * 4
        each = 6 * Dk * Dv if case["T"] == 1 else 6 * Dk * Dv + 4 * CHUNK * (Dk + Dv) // 2
        bytes_ = n * (wide + H * Dv) * es + 2 * ends
        if case["train"]:
            bytes_, each = bytes_ + n * (wide + H * Dv) * es + 2 * ends, each * 3
        return dict(bytes=bytes_, flops=n * H * each)
    es, ts, R, V, K = 4 if case["dtype"] == "f32" else 2, 4 if case["tdtype"] == "f32" else 2, case["R"], case["V"], case["K"]
    return dict(bytes=R * (V * es * (2 if case["train"] else 1) + K * (4 + ts) + 12), flops=R * V * (8 if case["train"] else 4))


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def _exact_embed(s, case):
    ids = s["ids"].long()
    at = torch.where(ids < 0, case["V"], ids)       # a row of zeros behind the table
    E = torch.cat((s["E"].double(), torch.zeros((1, case["D"]), dtype=torch.float64, device="cuda")))
    out = dict(Y=E.index_select(0, at).mul_(s["scale"]))
    if case["train"]:
        dE = torch.zeros((case["V"] + 1, case["D"]), dtype=torch.float64, device="cuda")
        order = at.argsort(stable=True)
        for piece in order.split(16384):
            dE.index_add_(0, at[piece], s["dY"][piece].double())
        out["dE"] = dE[:-1] * s["scale"] + (s["dE"].double() if case["add"] else 0)
    return out


def _exact_gdr(s, case):
    """Step by step, as the recurrence is written."""
    T, B, Hk, H, Dk, Dv = (case[k] for k in ("T", "B", "Hk", "H", "Dk", "Dv"))
    q, k, v, f, b = (t.double() for t in s["parts"])
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"].long()
    live = (torch.arange(T, device="cuda").unsqueeze(1) < n).double()
    lq, lk = (torch.sqrt(torch.linalg.vecdot(t, t) + EPS).unsqueeze(-1) for t in (q, k))
    share = torch.arange(H, device="cuda") // (H // Hk)
    qh, kh = ((t / l)[:, :, share] for t, l in ((q, lq), (k, lk)))
    a = torch.sigmoid(f) * live.unsqueeze(2) + (1 - live.unsqueeze(2))
    w = torch.sigmoid(b) * live.unsqueeze(2)
    S, kept, o = s["S0"].double(), [], []
    for t in range(T):
        kt, at, wt = kh[t].unsqueeze(3), a[t].view(B, H, 1, 1), w[t].view(B, H, 1, 1)
        if case["train"]:
            kept.append(S)
        S = at * S
        S = S + kt * (wt * (v[t].unsqueeze(2) - (kt * S).sum(2, keepdim=True)))
        o.append((qh[t].unsqueeze(3) * S).sum(2) * (s["scale"] * live[t].view(B, 1, 1)))
    out = dict(o=torch.stack(o), ST=S)
    if not case["train"]:
        return out
    kept.append(S)
    do = s["do"].double() * live.view(T, B, 1, 1)
    g = [torch.zeros_like(x) for x in (qh, kh, v, f, b)]
    dS = s["dST"].double()
    for t in range(T - 1, -1, -1):
        kt, at, wt, dot = kh[t].unsqueeze(3), a[t].view(B, H, 1, 1), w[t].view(B, H, 1, 1), do[t].unsqueeze(2)
        dS = dS + s["scale"] * qh[t].unsqueeze(3) * dot
        g[0][t] = s["scale"] * (kept[t + 1] * dot).sum(3)
        faded = at * kept[t]
        e = v[t].unsqueeze(2) - (kt * faded).sum(2, keepdim=True)
        through = (dS * kt).sum(2, keepdim=True)
        de = wt * through
        g[4][t] = (through * e).sum((2, 3)) * w[t] * (1 - w[t])
        g[1][t] = (dS * (wt * e)).sum(3) - (faded * de).sum(3)
        g[2][t] = de.squeeze(2)
        dS = dS - kt * de
        g[3][t] = (dS * kept[t]).sum((2, 3)) * a[t] * torch.sigmoid(-f[t]) * live[t].unsqueeze(1)
        dS = at * dS
    found = []
    for d, x, l in ((g[0], q, lq), (g[1], k, lk)):
        d = torch.zeros_like(x).index_add_(2, share, d) * live.view(T, B, 1, 1)
        found.append(d / l - x * (torch.linalg.vecdot(x, d).unsqueeze(-1) / l ** 3))
    return dict(out, dq=found[0], dk=found[1], dv=g[2], df=g[3], db=g[4], dS0=dS)


def _exact_distill(s, case):
    loss, dZ = [], []
    T, alpha, at = case["T"], case["alpha"], s["ids"].long()
    for rows in torch.arange(case["R"], device="cuda").split(max(1, (1 << 26) // case["V"])):
        Z = s["Z"][rows].double()
        logp = torch.log_softmax(s["t"][rows].double() / T, 1)
        logq = torch.log_softmax(Z / T, 1)
        target = torch.zeros_like(Z).scatter_add_(1, at[rows], logp.exp())
        one = alpha * T * T * torch.linalg.vecdot(logp.exp(), logp - logq.gather(1, at[rows]))
        grad = alpha * T * (logq.exp() - target)
        if s["labels"] is not None:
            y = s["labels"][rows].long()
            logh = torch.log_softmax(Z, 1)
            with_label = (y >= 0).double()
            one -= (1 - alpha) * with_label * logh.gather(1, y.clamp_min(0).unsqueeze(1)).squeeze(1)
            grad += (1 - alpha) * with_label.unsqueeze(1) * (logh.exp() - (torch.arange(case["V"], device="cuda") == y.unsqueeze(1)).double())
        loss.append(one)
        if case["train"]:
            dZ.append(grad * s["dloss"][rows].double().unsqueeze(1))
    return dict(loss=torch.cat(loss), dZ=torch.cat(dZ)) if case["train"] else dict(loss=torch.cat(loss))


def exact(case, seed):
    s = prepare(case, seed)
    return dict(embed=_exact_embed, gdr=_exact_gdr, distill=_exact_distill)[case["family"]](s, case)
