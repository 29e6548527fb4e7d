"""Embedding, gated delta rule and distillation loss in dry-run mode: what the entry points accept, what they refuse, what they would
launch, and the workspaces they ask for, without a GPU."""
import ctypes as C
import inspect

import pytest
import torch

import dryrun as D
from paper_2203_05705_amd import binding as ard
from test_host_calls import STREAM, fake, fake_ws
from test_host_recurrent import strided

NAN, INF = float("nan"), float("inf")
INT = torch.int32


# ---- embedding -------------------------------------------------------------------------------

def _embed_args(heap, **change):
    a = dict(dtype=ard.BF16, wdtype=ard.F32, R=5, V=9, D=24, ids=heap(64), E=heap(4096), lde=24, scale=1.0, Y=heap(4096), ldy=24, stream=None)
    a.update(change)
    return a


def _embed_bwd_args(heap, **change):
    a = dict(dtype=ard.BF16, wdtype=ard.F32, R=5, V=9, D=24, ids=heap(64), dY=heap(4096), lddy=24, scale=1.0, beta=0.0, dE=heap(4096), lddE=24,
             ws=heap(1 << 20), ws_bytes=1 << 20, stream=None)
    a.update(change)
    return a


SIZES = ((dict(dtype=5), -3), (dict(wdtype=-1), -3), (dict(dtype=ard.F32, wdtype=ard.BF16), -3), (dict(R=0), -2), (dict(V=0), -2), (dict(D=-1), -2),
         (dict(R=(1 << 30) + 1), -2), (dict(V=(1 << 28) + 1), -2), (dict(D=(1 << 24) + 1), -2))


def test_embedding_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        good = ({}, dict(wdtype=ard.BF16), dict(dtype=ard.F32), dict(R=1, V=1, D=1, lde=1, ldy=1), dict(E=heap(64) + 4, Y=heap(64) + 2, ids=heap(64) + 4), dict(lde=1 << 40, ldy=1 << 40),
                dict(R=1 << 30, V=1 << 28, D=1 << 24, lde=1 << 24, ldy=1 << 24), dict(scale=INF))
        for change in good:
            assert lib.ard_embed_fwd(*_embed_args(heap, **change).values()) == 0, change
            assert D.launches(lib) == (1, ["embed_fwd_kernel"])
        for change, code in SIZES + ((dict(lde=23), -2), (dict(ldy=23), -2), (dict(ids=None), -1), (dict(E=None), -1), (dict(Y=None), -1), (dict(Y=heap(64) + 1), -1),
                                     (dict(E=heap(64) + 2), -1), (dict(ids=heap(64) + 2), -1)):
            assert lib.ard_embed_fwd(*_embed_args(heap, **change).values()) == code and lib.ard_last_error(), change
        assert D.launches(lib)[0] == 0


def test_embedding_gradient_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        # more tokens than one row's lanes sum at once: a launch for the pieces
        for R, kernels in ((1, ["embed_sort_kernel", "embed_bwd_kernel"]), (32, ["embed_sort_kernel", "embed_bwd_kernel"]),
                           (33, ["embed_sort_kernel", "embed_pieces_kernel", "embed_bwd_kernel"])):
            for change in ({}, dict(beta=1.0), dict(wdtype=ard.BF16), dict(dtype=ard.F32)):
                assert lib.ard_embed_bwd(*_embed_bwd_args(heap, R=R, **change).values()) == 0, change
                assert D.launches(lib) == (len(kernels), kernels)
        need = lib.ard_embed_workspace_bytes(700, 50, 24)
        assert need >= (700 + 51) * 4 and lib.ard_embed_bwd(*_embed_bwd_args(heap, R=700, V=50, ws_bytes=need).values()) == 0
        D.launches(lib)
        for change, code in SIZES + ((dict(lddy=23), -2), (dict(lddE=23), -2), (dict(beta=0.5), -1), (dict(beta=NAN), -1), (dict(ids=None), -1), (dict(dY=None), -1),
                                     (dict(dE=None), -1), (dict(dY=heap(64) + 1), -1), (dict(R=700, V=50, ws_bytes=need - 1), -4), (dict(ws=None), -4), (dict(ws=heap(64) + 1), -4)):
            assert lib.ard_embed_bwd(*_embed_bwd_args(heap, **change).values()) == code and lib.ard_last_error(), change
        assert D.launches(lib)[0] == 0
        for sizes in ((0, 5, 5), (5, 0, 5), (5, 5, -1), ((1 << 30) + 1, 5, 5)):
            assert lib.ard_embed_workspace_bytes(*sizes) == 0


def test_pieces_of_the_most_tokens_have_a_grid():
    """HIP counts the threads along an axis of a grid in 32 bits."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for R in (33, 1 << 25, (1 << 25) + 1, 1 << 29, 1 << 30):
            need = lib.ard_embed_workspace_bytes(R, 9, 24)
            assert lib.ard_embed_bwd(*_embed_bwd_args(heap, R=R, ws_bytes=need).values()) == 0
            blocks, piece, threads = (int(v) for v in next(i for i in D.instances(lib) if i.startswith("embed_pieces_kernel")).split("<")[1][:-1].split(","))
            assert blocks * threads < 1 << 32 and piece * blocks >= min(R, 1 << 25)


# ---- gated delta rule ------------------------------------------------------------------------

def _steps(*all_):
    return (ard.CSteps * len(all_))(*(ard.CSteps(*s) for s in all_))


def _gdr_sizes(**change):
    a = dict(dtype=ard.BF16, T=100, B=3, Hk=2, H=4, Dk=40, Dv=50)
    a.update({k: v for k, v in change.items() if k in a})
    return a


def _gdr_in(heap, s, off=0):
    """The five inputs, contiguous."""
    wide = [s["Hk"] * s["Dk"]] * 2 + [s["H"] * s["Dv"]] + [s["H"]] * 2
    return _steps(*((heap(4096) + off, w * s["B"], w) for w in wide))


def _gdr_args(heap, **change):
    s = _gdr_sizes(**change)
    wide = s["H"] * s["Dv"]
    a = dict(s, inputs=_gdr_in(heap, s), scale=1.0, eps=1e-6, S0=heap(4096), lengths=heap(64), o=_steps((heap(4096), wide * s["B"], wide)), ST=heap(4096), ckpt=heap(4096),
             ws=heap(1 << 20), ws_bytes=1 << 40, stream=None)
    a.update(change)
    return a


def _gdr_bwd_args(heap, **change):
    s = _gdr_sizes(**change)
    wide = s["H"] * s["Dv"]
    a = dict(s, inputs=_gdr_in(heap, s), scale=1.0, eps=1e-6, lengths=heap(64), ckpt=heap(4096), do=_steps((heap(4096), wide * s["B"], wide)), dST=heap(4096), grads=_gdr_in(heap, s),
             dS0=heap(4096), ws=heap(1 << 20), ws_bytes=1 << 40, stream=None)
    a.update(change)
    return a


BACK = ["gdr_prep_kernel", "gdr_rows_kernel", "gdr_back_kernel", "gdr_grads_kernel"]
GDR_SIZES = ((dict(dtype=7), -3), (dict(T=0), -2), (dict(B=0), -2), (dict(Hk=0), -2), (dict(H=-1), -2), (dict(Dk=0), -2), (dict(Dv=0), -2), (dict(Hk=3), -2), (dict(Dk=129), -6),
             (dict(Dv=129), -6), (dict(T=(1 << 30) + 1), -2), (dict(B=1 << 19), -2))


def test_delta_rule_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        assert lib.ard_gdr_chunk() == ard.GDR_CHUNK == 64
        for T in (1, 2, 8, 9, 63, 64, 65, 1000):
            for change in ({}, dict(dtype=ard.F32), dict(S0=None), dict(ST=None), dict(ckpt=None), dict(lengths=None), dict(Dk=128, Dv=128), dict(Dk=1, Dv=1, Hk=4)):
                assert lib.ard_gdr_fwd(*_gdr_args(heap, T=T, **change).values()) == 0, change
                n, names = D.launches(lib)
                assert names == (["gdr_steps_kernel"] if T <= 8 else names) and n == (1 if T <= 8 else len(names)) and names[-1] in ("gdr_steps_kernel", "gdr_fwd_kernel")
                assert lib.ard_gdr_bwd(*_gdr_bwd_args(heap, T=T, **{k: v for k, v in change.items() if k in ("dtype", "lengths", "Dk", "Dv", "Hk")}).values()) == 0
                assert D.launches(lib)[1][-1] == "gdr_grads_kernel"
        assert lib.ard_gdr_bwd(*_gdr_bwd_args(heap, dST=None, dS0=None).values()) == 0
        D.launches(lib)
        more = ((dict(eps=0.0), -1), (dict(eps=INF), -1), (dict(eps=NAN), -1), (dict(scale=NAN), -1), (dict(scale=-INF), -1), (dict(inputs=None), -1), (dict(lengths=heap(64) + 2), -1),
                (dict(ckpt=heap(64) + 2), -1), (dict(ws=None), -4), (dict(ws=heap(64) + 8), -4), (dict(ws_bytes=100), -4))
        for change, code in GDR_SIZES + more + ((dict(o=None), -1), (dict(o=_steps((None, 1, 1))), -1), (dict(o=_steps((heap(64) + 1, 1, 1))), -1), (dict(S0=heap(64) + 2), -1),
                                                (dict(ST=heap(64) + 1), -1)):
            assert lib.ard_gdr_fwd(*_gdr_args(heap, **change).values()) == code and lib.ard_last_error(), change
        for change, code in GDR_SIZES + more + ((dict(do=None), -1), (dict(grads=None), -1), (dict(ckpt=None), -1), (dict(dST=heap(64) + 2), -1), (dict(dS0=heap(64) + 2), -1)):
            assert lib.ard_gdr_bwd(*_gdr_bwd_args(heap, **change).values()) == code and lib.ard_last_error(), change
        for i in range(5):
            a = _gdr_args(heap)
            a["inputs"][i].p = None
            assert lib.ard_gdr_fwd(*a.values()) == -1
            a = _gdr_args(heap)
            a["inputs"][i].p += 1
            assert lib.ard_gdr_fwd(*a.values()) == -1
            a = _gdr_bwd_args(heap)
            a["grads"][i].p = None
            assert lib.ard_gdr_bwd(*a.values()) == -1
        assert D.launches(lib)[0] == 0


def test_an_eps_whose_reciprocal_is_no_number_is_refused():
    """A key of zeros has the reciprocal length 1 / sqrt(eps); the product of two of them and a scale has to stay a number, as it meets a product of zeros."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for call, args in ((lib.ard_gdr_fwd, _gdr_args), (lib.ard_gdr_bwd, _gdr_bwd_args)):
            for eps in (1e-45, 1e-39, 1e-35, 2.0 ** -100 * 0.999):
                assert call(*args(heap, eps=eps).values()) == -1 and lib.ard_last_error(), eps
            for eps in (2.0 ** -100, 1e-30, 1e-12, 1.0):
                assert call(*args(heap, eps=eps).values()) == 0, eps


@pytest.mark.parametrize("dtype", [ard.F32, ard.BF16])
def test_delta_rule_workspaces(dtype):
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for T, B, Hk, H, Dk, Dv in ((1, 1, 1, 1, 1, 1), (8, 2, 1, 3, 64, 64), (9, 2, 1, 3, 64, 64), (64, 2, 2, 2, 65, 16), (65, 1, 1, 8, 128, 128), (16384, 1, 8, 8, 128, 128)):
            sizes = dict(dtype=dtype, T=T, B=B, Hk=Hk, H=H, Dk=Dk, Dv=Dv)
            for back, call, args in ((0, lib.ard_gdr_fwd, _gdr_args), (1, lib.ard_gdr_bwd, _gdr_bwd_args)):
                need = lib.ard_gdr_workspace_bytes(*sizes.values(), back)
                assert (need > 0) == bool(back or T > 8)
                assert call(*args(heap, **sizes, ws_bytes=need).values()) == 0
                if need:
                    assert call(*args(heap, **sizes, ws_bytes=need - 1).values()) == -4
        # a single step needs none at all
        assert lib.ard_gdr_fwd(*_gdr_args(heap, dtype=dtype, T=1, ws=None, ws_bytes=0).values()) == 0
        for change in (dict(T=0), dict(Dk=129), dict(Hk=3), dict(B=1 << 20)):
            assert lib.ard_gdr_workspace_bytes(*_gdr_sizes(dtype=dtype, **change).values(), 1) == 0
        # steps beyond 32-bit offsets, and the largest grids
        far = 1 << 33
        s = _gdr_sizes(dtype=dtype)
        assert lib.ard_gdr_fwd(*_gdr_args(heap, dtype=dtype, inputs=_steps(*((heap(64), far, 1 << 40) for _ in range(5)))).values()) == 0
        assert lib.ard_gdr_fwd(*_gdr_args(heap, dtype=dtype, B=1 << 18, H=4, T=128).values()) == 0
        assert s["T"] == 100


@pytest.mark.parametrize("dtype,T,B,Hk,H,Dk,Dv,back,segments", [
    (ard.F32, 4096, 2, 4, 4, 64, 128, 1, 11), (ard.F32, 4096, 4, 4, 4, 60, 64, 1, 8), (ard.F32, 2048, 4, 8, 8, 64, 64, 1, 8),   # LDS holds the operands of one workgroup
    (ard.BF16, 4096, 2, 8, 8, 128, 128, 1, 8), (ard.BF16, 16384, 1, 8, 8, 128, 128, 1, 16),
    (ard.BF16, 4096, 4, 8, 16, 64, 64, 1, 4), (ard.BF16, 16384, 1, 8, 8, 128, 128, 0, 16), (ard.F32, 4096, 4, 4, 4, 64, 64, 0, 13)])      # two, and their registers allow no more
def test_segments_go_by_what_a_compute_unit_holds_of_their_sums(dtype, T, B, Hk, H, Dk, Dv, back, segments):
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        sizes = dict(dtype=dtype, T=T, B=B, Hk=Hk, H=H, Dk=Dk, Dv=Dv)
        call, args = (lib.ard_gdr_bwd, _gdr_bwd_args) if back else (lib.ard_gdr_fwd, _gdr_args)
        assert call(*args(heap, **sizes, ws_bytes=lib.ard_gdr_workspace_bytes(*sizes.values(), back)).values()) == 0
        sums = next(i for i in D.instances(lib) if i.startswith("gdr_back_kernel<" if back else "gdr_fwd_kernel<"))
        workgroups, n, span = (int(v) for v in sums.split("<")[1][:-1].split(","))
        groups = -(-(128 if Dv > 64 else 64) // 64) if back else -(-Dv // 64)
        assert n == segments == -(-(-(-T // 64)) // span) and workgroups == B * H * (groups + (2 if Dk > 64 else 1)) * (n - 1)


# ---- distillation ----------------------------------------------------------------------------

def _distill_args(heap, **change):
    a = dict(dtype=ard.BF16, tdtype=ard.F32, R=4, V=100, K=7, Z=heap(4096), ldz=100, ids=heap(256), t=heap(256), labels=heap(64), temperature=2.0, alpha=0.5, dloss=heap(64),
             loss=heap(64), stats=heap(64), dZ=heap(4096), lddz=100, stream=None)
    a.update(change)
    return a


def _distill_bwd_args(heap, **change):
    a = dict(dtype=ard.BF16, tdtype=ard.F32, R=4, V=100, K=7, Z=heap(4096), ldz=100, ids=heap(256), t=heap(256), labels=heap(64), temperature=2.0, alpha=0.5, stats=heap(64),
             dloss=heap(64), dZ=heap(4096), lddz=100, stream=None)
    a.update(change)
    return a


def test_distillation_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for change in ({}, dict(tdtype=ard.BF16), dict(dtype=ard.F32), dict(labels=None), dict(dloss=None), dict(K=0, ids=None, t=None), dict(alpha=0.0, ids=None, t=None),
                       dict(alpha=1.0), dict(R=1, V=1, K=1, ldz=1, lddz=1), dict(K=1024), dict(V=1 << 30, ldz=1 << 30, lddz=1 << 30), dict(R=(1 << 31) - 1),
                       dict(Z=heap(64) + 2, dZ=heap(64) + 6), dict(ldz=1 << 40, lddz=1 << 40), dict(temperature=1e-3), dict(temperature=4.0), dict(temperature=1.0)):
            assert lib.ard_distill_fwd(*_distill_args(heap, **change).values()) == 0, change
            assert lib.ard_distill_bwd(*_distill_bwd_args(heap, **change).values()) == 0, change
            assert D.launches(lib)[0] == 2
        assert lib.ard_distill_fwd(*_distill_args(heap, dZ=None, lddz=0).values()) == 0
        D.launches(lib)
        both = ((dict(dtype=5), -3), (dict(tdtype=-1), -3), (dict(dtype=ard.F32, tdtype=ard.BF16), -3), (dict(R=0), -2), (dict(V=0), -2), (dict(K=-1), -2),
                (dict(V=(1 << 30) + 1, ldz=1 << 31, lddz=1 << 31), -2), (dict(K=1025), -6), (dict(ldz=99), -2), (dict(lddz=99), -2), (dict(temperature=0.0), -1),
                (dict(temperature=-1.0), -1), (dict(temperature=INF), -1), (dict(temperature=NAN), -1), (dict(alpha=-0.1), -1), (dict(alpha=1.1), -1), (dict(alpha=NAN), -1),
                (dict(Z=None), -1), (dict(ids=None), -1), (dict(t=None), -1), (dict(Z=heap(64) + 1), -1), (dict(t=heap(64) + 2), -1), (dict(ids=heap(64) + 2), -1),
                (dict(labels=heap(64) + 1), -1), (dict(stats=None), -1), (dict(stats=heap(64) + 2), -1), (dict(dloss=heap(64) + 1), -1), (dict(dZ=heap(64) + 1), -1))
        for change, code in both + ((dict(loss=None), -1), (dict(loss=heap(64) + 2), -1)):
            assert lib.ard_distill_fwd(*_distill_args(heap, **change).values()) == code and lib.ard_last_error(), change
        for change, code in both + ((dict(dZ=None), -1),):
            assert lib.ard_distill_bwd(*_distill_bwd_args(heap, **change).values()) == code and lib.ard_last_error(), change
        # in the logits' place, but rows of another distance would lie over each other
        for call, a in ((lib.ard_distill_fwd, _distill_args(heap)), (lib.ard_distill_bwd, _distill_bwd_args(heap))):
            D.launches(lib)
            a["dZ"] = a["Z"]
            assert call(*a.values()) == 0
            a["lddz"] = 104
            assert call(*a.values()) == -1 and D.launches(lib)[0] == 1
            a["R"] = 1
            assert call(*a.values()) == 0


def test_temperatures_whose_square_or_reciprocal_is_no_number_are_refused():
    """T^2 weighs the loss and log2(e) / T the logits: both are normal fp32 numbers from 2^-60 to 2^60."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for call, args in ((lib.ard_distill_fwd, _distill_args), (lib.ard_distill_bwd, _distill_bwd_args)):
            for T in (1e-45, 1e-39, 1e-30, 2.0 ** -60 * 0.999, 2.0 ** 60 * 1.001, 1e20, 3e38):
                for alpha in (0.0, 0.5, 1.0):
                    assert call(*args(heap, temperature=T, alpha=alpha).values()) == -1 and lib.ard_last_error(), T
            for T in (2.0 ** -60, 1e-3, 100.0, 2.0 ** 60):
                assert call(*args(heap, temperature=T).values()) == 0, T


@pytest.mark.parametrize("R", [1, 700, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, 1 << 30, (1 << 31) - (1 << 20), (1 << 31) - (1 << 20) + 1, (1 << 31) - 1])
def test_the_most_rows_of_logits_have_a_grid(R):
    """A workgroup for every row; HIP counts the threads along an axis of a grid in 32 bits and takes 65535 workgroups along its second."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for V in (100, 200000):
            for call, args in ((lib.ard_distill_fwd, _distill_args), (lib.ard_distill_bwd, _distill_bwd_args)):
                assert call(*args(heap, R=R, V=V, ldz=V, lddz=V).values()) == 0
                x, y, threads = (int(v) for v in D.instances(lib)[0].split("<")[1][:-1].split(","))
                assert 0 < x and x * threads < 1 << 32 and 0 < y <= 65535 and R <= x * y < R + x


# ---- through the binding ---------------------------------------------------------------------

def test_calls_of_the_binding():
    """Shapes of what a call makes by itself or finds, on tensors without memory."""
    ws = fake_ws(1 << 28)
    with D.dry_run() as lib:
        ids, E = fake(5, 3, dtype=INT), fake(50, 24)
        Y = ard.embed_fwd(ids, E, out=fake(5, 3, 24, dtype=torch.bfloat16), stream=STREAM)
        assert Y.dtype == torch.bfloat16 and D.launches(lib)[0] == 1
        dE = ard.embed_bwd(ids, Y, 50, out=E, ws=ws, stream=STREAM)
        assert dE is E and D.launches(lib)[0] == 2
        table = strided((50, 24), (30, 1))
        assert ard.embed_bwd(ids, strided((15, 24), (40, 1)), 50, beta=1, out=table, ws=ws, stream=STREAM) is table
        D.launches(lib)
        q, k, v, f, b = (strided((70, 3, *shape), (600, 200, *inner)) for shape, inner in (((2, 20), (20, 1)), ((2, 20), (20, 1)), ((4, 16), (16, 1)), ((4,), (1,)), ((4,), (1,))))
        o, S, ck = fake(70, 3, 4, 16), fake(3, 4, 20, 16), fake(2, 3, 4, 20, 16)
        got = ard.gdr_fwd(q, k, v, f, b, S, fake(3, dtype=INT), out=(o, S, ck), ws=ws, stream=STREAM)
        assert got[0] is o and got[1] is S and got[2] is ck
        assert D.launches(lib)[1][-1] == "gdr_fwd_kernel"
        grads = [strided(t.shape, t.stride()) for t in (q, k, v, f, b)]
        assert len(ard.gdr_bwd(q, k, v, f, b, o, ck, S, out=(*grads, S), ws=ws, stream=STREAM)) == 6
        assert D.launches(lib)[1][-1] == "gdr_grads_kernel"
        one = [strided((1, *t.shape[1:]), t.stride()) for t in (q, k, v, f, b)]
        assert ard.gdr_fwd(*one, S, train=False, out=(fake(1, 3, 4, 16), S, None), stream=STREAM)[2] is None
        assert D.launches(lib) == (1, ["gdr_steps_kernel"])
        Z, t, tid, y, loss, stats = fake(6, 90), fake(6, 4), fake(6, 4, dtype=INT), fake(6, dtype=INT), fake(6), fake(6, 3)
        got = ard.distill_fwd(Z, tid, t, labels=y, temperature=2, alpha=0.5, grad=True, out=(loss, stats, Z), stream=STREAM)
        assert got[0] is loss and got[2] is Z and D.launches(lib)[0] == 1
        assert ard.distill_fwd(Z, None, None, labels=y, alpha=0, out=(loss, stats, None), stream=STREAM)[2] is None
        assert ard.distill_bwd(Z, tid, t, stats, fake(6), labels=y, out=Z, stream=STREAM) is Z and D.launches(lib)[0] == 2


def test_what_the_binding_refuses():
    ws = fake_ws()
    kw = dict(stream=STREAM)
    ids, E, Y = fake(6, dtype=INT), fake(50, 24), fake(6, 24)
    z = [fake(9, 2, 2, 8), fake(9, 2, 2, 8), fake(9, 2, 4, 5), fake(9, 2, 4), fake(9, 2, 4)]
    out, ck, S = (fake(9, 2, 4, 5), fake(2, 4, 8, 5), fake(1, 2, 4, 8, 5)), fake(1, 2, 4, 8, 5), fake(2, 4, 8, 5)
    Z, t, tid, loss = fake(6, 90), fake(6, 4), fake(6, 4, dtype=INT), (fake(6), fake(6, 3), None)

    def gdr(i, other, **more):
        return lambda: ard.gdr_fwd(*z[:i], other, *z[i + 1:], out=out, ws=ws, **{**kw, **more})
    bad = (ValueError, AssertionError, TypeError, IndexError)
    with D.dry_run() as lib:
        for call in [
                lambda: ard.embed_fwd(fake(6), E, out=Y, **kw), lambda: ard.embed_fwd(fake(6, dtype=torch.int64), E, out=Y, **kw),
                lambda: ard.embed_fwd(ids, fake(50), out=Y, **kw), lambda: ard.embed_fwd(ids, E, out=fake(5, 24), **kw), lambda: ard.embed_fwd(ids, E, out=fake(6, 23), **kw),
                lambda: ard.embed_fwd(ids, E, dtype=torch.bfloat16, out=Y, **kw), lambda: ard.embed_fwd(ids, fake(50, 24, dtype=torch.float16), out=Y, **kw),
                lambda: ard.embed_fwd(ids, strided((50, 24), (1, 50)), out=Y, **kw), lambda: ard.embed_fwd(ids, E, out=strided((6, 24), (20, 1)), **kw),
                lambda: ard.embed_fwd(ids, torch.zeros(50, 24), out=Y, **kw), lambda: ard.embed_fwd(torch.zeros(6, dtype=INT), E, out=Y, **kw),
                lambda: ard.embed_bwd(ids, Y, 0, out=E, ws=ws, **kw), lambda: ard.embed_bwd(ids, Y, 49, out=E, ws=ws, **kw), lambda: ard.embed_bwd(ids, fake(5, 24), 50, out=E, ws=ws, **kw),
                lambda: ard.embed_bwd(ids, Y, 50, beta=1.0, ws=ws, **kw), lambda: ard.embed_bwd(ids, Y, 50, dtype=torch.bfloat16, out=E, ws=ws, **kw),
                lambda: ard.embed_bwd(ids, Y, 50, out=strided((50, 24), (20, 1)), ws=ws, **kw),
                gdr(0, fake(9, 2, 16)), gdr(0, fake(9, 2, 2, 8, dtype=torch.bfloat16)), gdr(1, fake(9, 2, 2, 7)), gdr(1, fake(8, 2, 2, 8)), gdr(2, fake(9, 2, 4, 0)), gdr(3, fake(9, 2, 4, 1)),
                gdr(4, fake(9, 2, 3)), gdr(0, strided((9, 2, 2, 8), (64, 32, 16, 1))), gdr(2, strided((9, 2, 4, 5), (40, 20, 5, 2))), gdr(0, torch.zeros(9, 2, 2, 8)),
                gdr(0, z[0], S0=fake(2, 4, 8, 4)), gdr(0, z[0], S0=strided((2, 4, 8, 5), (40, 80, 5, 1))), gdr(0, z[0], lengths=fake(3, dtype=INT)), gdr(0, z[0], lengths=fake(2)),
                lambda: ard.gdr_fwd(*z, out=(strided((9, 2, 4, 5), (20, 10, 5, 1)), *out[1:]), ws=ws, **kw), lambda: ard.gdr_fwd(*z, out=(out[0], out[1]), ws=ws, **kw),
                lambda: ard.gdr_fwd(*z, out=(*out[:2], fake(2, 2, 4, 8, 5)), ws=ws, **kw),
                lambda: ard.gdr_bwd(*z, out[0], None, out=(*z, S), ws=ws, **kw), lambda: ard.gdr_bwd(*z, fake(9, 2, 4, 6), ck, out=(*z, S), ws=ws, **kw),
                lambda: ard.gdr_bwd(*z, out[0], fake(2, 2, 4, 8, 5), out=(*z, S), ws=ws, **kw), lambda: ard.gdr_bwd(*z, out[0], ck, out=z, ws=ws, **kw),
                lambda: ard.gdr_bwd(*z, out[0], ck, out=(strided((9, 2, 2, 8), (0, 16, 8, 1)), *z[1:], S), ws=ws, **kw),
                lambda: ard.distill_fwd(Z, tid, None, out=loss, **kw), lambda: ard.distill_fwd(Z, None, t, out=loss, **kw), lambda: ard.distill_fwd(Z, fake(6, 3, dtype=INT), t, out=loss, **kw),
                lambda: ard.distill_fwd(Z, fake(5, 4, dtype=INT), fake(5, 4), out=loss, **kw), lambda: ard.distill_fwd(Z, fake(6, 4), t, out=loss, **kw), lambda: ard.distill_fwd(strided((6, 90), (1, 6)), tid, t, out=loss, **kw),
                lambda: ard.distill_fwd(Z, tid, t, labels=fake(6), out=loss, **kw), lambda: ard.distill_fwd(Z, tid, t, labels=fake(5, dtype=INT), out=loss, **kw),
                lambda: ard.distill_fwd(Z, tid, t, dloss=fake(5), out=(*loss[:2], Z), **kw), lambda: ard.distill_fwd(Z, tid, t, grad=True, out=(*loss[:2], fake(6, 89)), **kw),
                lambda: ard.distill_fwd(Z, tid, t, grad=True, out=(*loss[:2], fake(6, 90, dtype=torch.bfloat16)), **kw), lambda: ard.distill_fwd(Z, tid, t, out=(fake(5), loss[1], None), **kw),
                lambda: ard.distill_bwd(Z, tid, t, None, out=Z, **kw), lambda: ard.distill_bwd(Z, tid, t, fake(6, 2), out=Z, **kw), lambda: ard.distill_bwd(Z, tid, t, loss[1], out=fake(5, 90), **kw)]:
            with pytest.raises(bad):
                call()
        for call in [lambda: ard.embed_bwd(ids, Y, 50, beta=0.5, out=E, ws=ws, **kw), lambda: ard.embed_bwd(ids, Y, 50, out=E, ws=fake_ws(8), **kw),
                     gdr(0, z[0], eps=0.0), gdr(0, z[0], scale=NAN), gdr(1, z[1], eps=-1.0),
                     lambda: ard.gdr_fwd(fake(9, 2, 1, 129), fake(9, 2, 1, 129), fake(9, 2, 1, 5), fake(9, 2, 1), fake(9, 2, 1), out=(fake(9, 2, 1, 5), fake(2, 1, 129, 5), None), train=False,
                                         ws=ws, **kw),
                     lambda: ard.distill_fwd(Z, tid, t, temperature=0.0, out=loss, **kw), lambda: ard.distill_fwd(Z, tid, t, alpha=2.0, out=loss, **kw),
                     lambda: ard.distill_fwd(Z, fake(6, 1025, dtype=INT), fake(6, 1025), out=loss, **kw),
                     lambda: ard.distill_fwd(Z, tid, fake(6, 4, dtype=torch.bfloat16), out=loss, **kw)]:
            with pytest.raises(ard.ArdError):
                call()
        assert D.launches(lib)[0] == 0


def test_calls_without_rows():
    with D.dry_run() as lib:
        assert ard.embed_fwd(fake(0, dtype=INT), fake(5, 3), out=fake(0, 3), stream=STREAM).shape == (0, 3)
        assert ard.embed_bwd(fake(0, dtype=INT), fake(0, 3), 5, beta=1.0, out=fake(5, 3), stream=STREAM).shape == (5, 3)
        none = ard.distill_fwd(fake(0, 7), None, None, out=(fake(0), fake(0, 3), fake(0, 7)), grad=True, stream=STREAM)
        assert none[2].shape == (0, 7) and D.launches(lib)[0] == 0


def test_signatures_can_be_read():
    want = dict(
        embed_fwd="ids, E, scale=1.0, dtype=None, out=None, stream=None", embed_bwd="ids, dY, V, scale=1.0, beta=0.0, dtype=None, out=None, ws=None, stream=None",
        distill_fwd="Z, ids, t, labels=None, temperature=1.0, alpha=1.0, dloss=None, grad=None, out=None, stream=None",
        distill_bwd="Z, ids, t, stats, dloss=None, labels=None, temperature=1.0, alpha=1.0, out=None, stream=None",
        gdr_fwd="q, k, v, f, b, S0=None, lengths=None, scale=None, eps=1e-06, train=True, out=None, ws=None, stream=None",
        gdr_bwd="q, k, v, f, b, do, ckpt, dST=None, lengths=None, scale=None, eps=1e-06, out=None, ws=None, stream=None")
    for name, params in want.items():
        assert str(inspect.signature(getattr(ard, name))) == f"({params})", name
        assert getattr(ard, name).__doc__
    assert C.sizeof(ard.CSteps) == 24
