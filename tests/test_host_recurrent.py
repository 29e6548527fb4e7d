"""Layer norm, the gated linear recurrence and AdamW in dry-run mode: what the entry points accept, what they refuse, what they
would launch, and the workspaces they ask for, without a GPU."""
import ctypes as C
import inspect

import pytest
import torch

import dryrun as D
from paper_2203_05705_amd import binding as ard
from test_host_calls import STREAM, fake, fake_ws

BOTH = ard.IN_COMPACT | ard.OUT_COMPACT
_heap = D.FakeHeap()


def strided(shape, stride, dtype=torch.float32):
    """A tensor of these strides at an address nothing is mapped at."""
    n = (sum((s - 1) * t for s, t in zip(shape, stride)) + 1) * dtype.itemsize
    storage = torch._C._construct_storage_from_data_pointer(_heap(n), torch.device("cuda:0"), n)
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(dtype=dtype, size=torch.Size(shape), stride=stride, storage_offset=0, device=torch.device("cuda:0"), data_ptr=0, nbytes=n), storage)


# ---- layer norm ------------------------------------------------------------------------------

def _norm_args(heap, **change):
    a = dict(dtype=ard.BF16, wdtype=ard.F32, R=4, D=24, X=heap(4096), ldx=24, gamma=heap(4096), beta=heap(4096), eps=1e-5, Y=heap(4096), ldy=24,
             mean=heap(64), rstd=heap(64), flags=0, stream=None)
    a.update(change)
    return a


def _norm_bwd_args(heap, **change):
    a = dict(dtype=ard.BF16, wdtype=ard.F32, R=4, D=24, dY=heap(4096), lddy=24, X=heap(4096), ldx=24, gamma=heap(4096), mean=heap(64), rstd=heap(64),
             dX=heap(4096), lddx=24, dgamma=heap(4096), dbeta=heap(4096), flags=0, ws=heap(1 << 20), ws_bytes=1 << 20, stream=None)
    a.update(change)
    return a


def test_norm_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for change in ({}, dict(gamma=None), dict(beta=None), dict(wdtype=ard.BF16), dict(dtype=ard.F32), dict(flags=ard.OUT_COMPACT), dict(R=1, D=1, ldx=1, ldy=1),
                       dict(D=20, ldx=24, ldy=24, flags=ard.OUT_COMPACT), dict(X=heap(64) + 2, Y=heap(64) + 6), dict(ldx=1 << 40)):
            assert lib.ard_layer_norm_fwd(*_norm_args(heap, **change).values()) == 0, change
        assert D.launches(lib)[0] == 10
        for change, code in ((dict(dtype=5), -3), (dict(wdtype=-1), -3), (dict(dtype=ard.F32, wdtype=ard.BF16), -3), (dict(R=0), -2), (dict(D=-1), -2),
                             (dict(D=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31), -2), (dict(ldx=23), -2), (dict(ldy=0), -2),
                             (dict(D=20, ldx=20, ldy=20, flags=ard.OUT_COMPACT), -2), (dict(X=None), -1), (dict(Y=None), -1), (dict(mean=None), -1),
                             (dict(rstd=None), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(flags=ard.IN_COMPACT), -1),
                             (dict(X=heap(64) + 1), -1), (dict(gamma=heap(64) + 2), -1), (dict(mean=heap(64) + 2), -1)):
            assert lib.ard_layer_norm_fwd(*_norm_args(heap, **change).values()) == code and lib.ard_last_error(), change
        assert D.launches(lib)[0] == 0


def test_norm_backward_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        # few rows: one launch and no workspace; more: a second launch for the weights' gradients, if any are asked for
        for R, kernels in ((4, ["norm_bwd_few_kernel"]), (512, ["norm_bwd_few_kernel"]), (513, ["norm_bwd_kernel", "norm_weight_grad_kernel"])):
            for change in ({}, dict(dgamma=None), dict(dbeta=None), dict(gamma=None)):
                assert lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, R=R, **change).values()) == 0
                assert D.launches(lib) == (len(kernels), kernels)
            assert lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, R=R, dgamma=None, dbeta=None, ws=None, ws_bytes=0).values()) == 0
            assert D.launches(lib) == (1, kernels[:1])
            assert (lib.ard_layer_norm_workspace_bytes(R, 24) > 0) == (R > 512)
        assert lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, ws=None, ws_bytes=0).values()) == 0
        D.launches(lib)
        assert lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, D=20000, ldx=20000, lddy=20000, lddx=20000, ws_bytes=1 << 30).values()) == 0
        assert D.launches(lib) == (3, ["norm_bwd_long_kernel", "norm_bwd_cols_kernel", "norm_weight_grad_kernel"])
        need = lib.ard_layer_norm_workspace_bytes(600, 24)
        assert need > 0 and lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, R=600, ws_bytes=need).values()) == 0
        D.launches(lib)
        for change, code in ((dict(R=600, ws_bytes=need - 1), -4), (dict(R=600, ws=None), -4), (dict(lddy=23), -2), (dict(lddx=23), -2), (dict(dY=None), -1), (dict(dX=None), -1),
                             (dict(mean=None), -1), (dict(rstd=None), -1), (dict(D=20, lddx=23, flags=ard.OUT_COMPACT), -2), (dict(dX=heap(64) + 1), -1),
                             (dict(dgamma=heap(64) + 2), -1)):
            assert lib.ard_layer_norm_bwd(*_norm_bwd_args(heap, **change).values()) == code, change
        assert D.launches(lib)[0] == 0
        assert lib.ard_layer_norm_workspace_bytes(0, 5) == 0 and lib.ard_layer_norm_workspace_bytes(5, -1) == 0


def test_norm_backward_in_the_place_of_an_input_makes_its_sums_over_rows_first():
    """Sums over rows that are made from the inputs once more may not meet a dX that is stored meanwhile or before."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for place in ("dY", "X"):
            for R, n, kernels in ((4, 24, ["norm_bwd_few_kernel"] * 2), (512, 24, ["norm_bwd_few_kernel"] * 2), (513, 24, ["norm_bwd_kernel", "norm_weight_grad_kernel"]),
                                  (4, 20000, ["norm_bwd_cols_kernel", "norm_bwd_long_kernel", "norm_weight_grad_kernel"])):
                a = _norm_bwd_args(heap, R=R, D=n, ldx=n, lddy=n, lddx=n, ws_bytes=1 << 30)
                a["dX"] = a[place]
                assert lib.ard_layer_norm_bwd(*a.values()) == 0 and D.launches(lib) == (len(kernels), kernels)
                a.update(dgamma=None, dbeta=None)
                assert lib.ard_layer_norm_bwd(*a.values()) == 0 and D.launches(lib)[0] == 1
                a["lddx"] = n + 8   # rows that lie elsewhere than the input's, over each other
                assert lib.ard_layer_norm_bwd(*a.values()) == -1 and D.launches(lib)[0] == 0
                a["R"] = 1
                assert lib.ard_layer_norm_bwd(*a.values()) == 0 and D.launches(lib)[0] == 1
        a = _norm_args(heap)
        a["Y"] = a["X"]
        assert lib.ard_layer_norm_fwd(*a.values()) == 0 and D.launches(lib)[0] == 1
        a["ldy"] = 32
        assert lib.ard_layer_norm_fwd(*a.values()) == -1 and D.launches(lib)[0] == 0


@pytest.mark.parametrize("dtype", [ard.F32, ard.BF16])
def test_norm_takes_rows_of_every_length(dtype):
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for n in list(range(1, 140)) + [k + d for k in (512, 1024, 2048, 4096, 8192, 16384) for d in (-1, 0, 1)] + [1 << 20, 1 << 30]:
            a = _norm_args(heap, dtype=dtype, D=n, ldx=n, ldy=n, R=(1 << 31) - 1)
            assert lib.ard_layer_norm_fwd(*a.values()) == 0, n
            name = D.launches(lib)[1]
            assert name == (["norm_fwd_kernel"] if n <= 16384 else ["norm_fwd_long_kernel"]), n


def test_norm_gradients_of_the_longest_rows_have_a_grid():
    """HIP counts the threads along an axis of a grid in 32 bits; 16 of dgamma's and dbeta's columns a workgroup of 1024."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for n in (16385, (1 << 25) - 9, 1 << 25, (1 << 25) + 24, (1 << 29) + 5, 1 << 30):
            ws = lib.ard_layer_norm_workspace_bytes(2, n)
            a = _norm_bwd_args(heap, R=2, D=n, ldx=n, lddy=n, lddx=n, ws_bytes=ws)
            assert lib.ard_layer_norm_bwd(*a.values()) == 0
            x, y, threads = (int(v) for v in next(i for i in D.instances(lib) if i.startswith("norm_weight_grad_kernel")).split("<")[1][:-1].split(","))
            assert x * threads < 1 << 32 and 2 * n <= x * y * 16 < 2 * n + 16 * (y + 1), n


# ---- gated linear recurrence -------------------------------------------------------------------

def _glr_args(heap, **change):
    a = dict(dtype=ard.BF16, T=40, B=3, H=20, f=heap(1 << 16), v=heap(1 << 16), o=heap(1 << 16), z_t=60, z_b=20, c0=heap(256), len=heap(64), h=heap(1 << 16), h_t=60,
             h_b=20, cT=heap(256), ckpt=heap(1 << 16), flags=0, ws=None, ws_bytes=0, stream=None)
    a.update(change)
    return a


def _glr_bwd_args(heap, **change):
    a = dict(dtype=ard.BF16, T=40, B=3, H=20, f=heap(1 << 16), v=heap(1 << 16), o=heap(1 << 16), z_t=60, z_b=20, len=heap(64), ckpt=heap(1 << 16), dh=heap(1 << 16),
             dh_t=60, dh_b=20, dcT=heap(256), df=heap(1 << 16), dv=heap(1 << 16), do=heap(1 << 16), dz_t=60, dz_b=20, dc0=heap(256), flags=0, ws=None, ws_bytes=0,
             stream=None)
    a.update(change)
    return a


def test_recurrence_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for change in ({}, dict(o=None), dict(c0=None), dict(len=None), dict(cT=None), dict(ckpt=None), dict(flags=BOTH), dict(dtype=ard.F32), dict(H=19), dict(f=heap(64) + 2)):
            assert lib.ard_glr_fwd(*_glr_args(heap, **change).values()) == 0, change
            assert D.launches(lib) == (1, ["glr_fwd_kernel"])
        state = heap(256)
        assert lib.ard_glr_fwd(*_glr_args(heap, T=1, c0=state, cT=state).values()) == 0 and D.launches(lib) == (1, ["glr_step_kernel"])
        for change, code in ((dict(dtype=2), -3), (dict(T=0), -2), (dict(B=0), -2), (dict(H=-4), -2), (dict(T=(1 << 30) + 1), -2), (dict(H=(1 << 24) + 1), -2), (dict(f=None), -1),
                             (dict(v=None), -1), (dict(h=None), -1), (dict(flags=ard.OUT_COMPACT), -1), (dict(flags=64), -1), (dict(c0=state, cT=state), -1),
                             (dict(v=heap(64) + 1), -1), (dict(c0=heap(64) + 2), -1), (dict(len=heap(64) + 1), -1), (dict(B=1 << 30), -2)):
            assert lib.ard_glr_fwd(*_glr_args(heap, **change).values()) == code and lib.ard_last_error(), change
        assert D.launches(lib)[0] == 0


def test_recurrence_backward_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for change in ({}, dict(o=None, do=None), dict(dcT=None), dict(dc0=None), dict(len=None), dict(flags=BOTH), dict(dtype=ard.F32), dict(T=1), dict(dh_t=0, dh_b=0)):
            assert lib.ard_glr_bwd(*_glr_bwd_args(heap, **change).values()) == 0, change
            assert D.launches(lib) == (1, ["glr_bwd_kernel"])
        for change, code in ((dict(o=None), -1), (dict(do=None), -1), (dict(ckpt=None), -1), (dict(dh=None), -1), (dict(df=None), -1), (dict(dv=None), -1), (dict(T=-1), -2),
                             (dict(dh=heap(64) + 1), -1), (dict(dtype=9), -3)):
            assert lib.ard_glr_bwd(*_glr_bwd_args(heap, **change).values()) == code, change
        assert D.launches(lib)[0] == 0


@pytest.mark.parametrize("dtype", [ard.F32, ard.BF16])
def test_cut_sequences_ask_for_a_workspace(dtype):
    """Few channels and many steps: two launches and room for the segments' pairs; the same room serves compact channels."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for T, B, H in ((1000, 1, 10), (32768, 1, 1024), (4096, 3, 683), (1 << 20, 1, 1)):
            need = lib.ard_glr_workspace_bytes(dtype, T, B, H)
            assert need > 0
            for flags in (0, BOTH):
                a = _glr_args(heap, dtype=dtype, T=T, B=B, H=H, flags=flags, ws=heap(64), ws_bytes=need)
                assert lib.ard_glr_fwd(*a.values()) == 0
                assert D.launches(lib) == (2, ["glr_fwd_pairs_kernel", "glr_fwd_kernel"])
                a = _glr_bwd_args(heap, dtype=dtype, T=T, B=B, H=H, flags=flags, ws=heap(64), ws_bytes=need)
                assert lib.ard_glr_bwd(*a.values()) == 0
                assert D.launches(lib) == (2, ["glr_bwd_pairs_kernel", "glr_bwd_kernel"])
            a = _glr_args(heap, dtype=dtype, T=T, B=B, H=H, ws=heap(64), ws_bytes=16)
            assert lib.ard_glr_fwd(*a.values()) == -4 and b"workspace" in lib.ard_last_error()
            assert lib.ard_glr_fwd(*_glr_args(heap, dtype=dtype, T=T, B=B, H=H).values()) == -4
        for T, B, H in ((1, 1, 1), (64, 128, 1024), (16, 1, 4)):
            assert lib.ard_glr_workspace_bytes(dtype, T, B, H) == 0
        assert lib.ard_glr_workspace_bytes(7, 1000, 1, 10) == 0 and lib.ard_glr_workspace_bytes(dtype, 0, 1, 10) == 0
        assert lib.ard_glr_chunk() == ard.GLR_CHUNK


@pytest.mark.parametrize("dtype", [ard.F32, ard.BF16])
def test_recurrence_launches_a_workgroup_for_every_segment_of_every_lane(dtype):
    """The grids: as many wavefronts as the sequences' lanes fill, times the segments that the workspace has room for (a first pass of
    the forward direction: but the last); one workgroup more would read behind the workspace."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for T, B, H in ((1, 5, 20), (40, 3, 20), (64, 128, 1024), (100, 7, 3), (1000, 1, 10), (2500, 3, 64), (5000, 48, 22), (700, 20, 500), (32768, 1, 1024), (4099, 9, 131)):
            for flags in (0, BOTH):
                wide = -(-H // 8) * 8 if flags else H
                groups = {-(-B * wide // 64)} if dtype == ard.F32 or wide % 2 else {-(-B * wide // 64), -(-B * (wide // 2) // 64)}
                room = lib.ard_glr_workspace_bytes(dtype, T, B, H)
                kw = dict(dtype=dtype, T=T, B=B, H=H, flags=flags, ws=heap(64), ws_bytes=room)
                assert lib.ard_glr_fwd(*_glr_args(heap, **kw).values()) == 0
                assert lib.ard_glr_bwd(*_glr_bwd_args(heap, **kw).values()) == 0
                for launch in D.instances(lib):
                    name, (grid, of, segs) = launch.split("<")[0], (int(v) for v in launch.split("<")[1][:-1].split(","))
                    assert of in groups and grid == of * (segs - 1 if name == "glr_fwd_pairs_kernel" else segs), launch
                    assert segs == 1 or segs * 2 * B * H * 4 <= room, launch


# ---- AdamW ----------------------------------------------------------------------------------------

def _tensor(heap, n, bits=32, **change):
    s = ard.CAdamWTensor(n, heap(64), heap(64), heap(64), heap(64), heap(64) if bits == 8 else None, heap(64) if bits == 8 else None, None)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def _step(lib, tensors, bits=32, gdtype=ard.F32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1, count=None, scale=None):
    arr = (ard.CAdamWTensor * max(1, len(tensors)))(*tensors)
    return lib.ard_adamw_step(bits, gdtype, len(tensors) if count is None else count, arr if tensors else None, lr, b1, b2, eps, wd, step, scale, None)


def test_adamw_accepts_and_refuses():
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        t = _tensor(heap, 10)
        for bits in (32, 8):
            for gdtype in (ard.F32, ard.BF16):
                assert _step(lib, [_tensor(heap, 10, bits)], bits, gdtype) == 0 and D.launches(lib) == (1, ["adamw_kernel"])
        assert _step(lib, []) == 0 and _step(lib, [_tensor(heap, 0), ard.CAdamWTensor()]) == 0 and D.launches(lib)[0] == 0
        for kw, code in ((dict(bits=16), -1), (dict(gdtype=3), -3), (dict(count=-1), -2), (dict(lr=-1.0), -1), (dict(lr=float("nan")), -1), (dict(b1=1.0), -1), (dict(b2=-0.1), -1),
                         (dict(eps=0.0), -1), (dict(eps=float("inf")), -1), (dict(wd=-1.0), -1), (dict(step=0), -1), (dict(scale=heap(64) + 1), -1)):
            assert _step(lib, [t], **kw) == code and lib.ard_last_error(), kw
        assert _step(lib, [], count=3) == -1
        for bad, bits, code in ((_tensor(heap, -1), 32, -2), (_tensor(heap, 5, p=None), 32, -1), (_tensor(heap, 5, g=None), 32, -1), (_tensor(heap, 5, m=None), 32, -1),
                                (_tensor(heap, 5, 8, v_scale=None), 8, -1), (_tensor(heap, 5, 8), 32, -1), (_tensor(heap, 5, p=heap(64) + 2), 32, -1),
                                (_tensor(heap, 5, w=heap(64) + 1), 32, -1), (_tensor(heap, 5, 8, m_scale=heap(64) + 2), 8, -1)):
            assert _step(lib, [_tensor(heap, 10, bits), bad], bits) == code, bad
        assert D.launches(lib)[0] == 0


def test_adamw_deals_tensors_over_launches():
    """48 tensors a launch, none of empty tensors; a tensor of more workgroups than a launch may have is dealt to several."""
    with D.dry_run() as lib:
        heap = D.FakeHeap()
        for count, launches in ((1, 1), (48, 1), (49, 2), (97, 3)):
            assert _step(lib, [_tensor(heap, 5 + i) for i in range(count)]) == 0 and D.launches(lib)[0] == launches
        assert _step(lib, [_tensor(heap, 0 if i % 2 else 7) for i in range(96)]) == 0 and D.launches(lib)[0] == 1
        assert _step(lib, [_tensor(heap, 1 << 35)]) == 0 and D.launches(lib)[0] == 1
        assert _step(lib, [_tensor(heap, (1 << 35) + 1), _tensor(heap, 9)]) == 0 and D.launches(lib)[0] == 2
        t = [_tensor(heap, 300, 8) for _ in range(50)]
        outs = (C.c_void_p * 50)(*[heap(2048) for _ in range(50)])
        assert lib.ard_adamw_values(50, (ard.CAdamWTensor * 50)(*t), outs, outs, None) == 0 and D.launches(lib) == (2, ["adamw_values_kernel"] * 2)
        assert lib.ard_adamw_values(0, None, None, None, None) == 0
        assert lib.ard_adamw_values(50, (ard.CAdamWTensor * 50)(*t), None, outs, None) == -1
        outs[3] = None
        assert lib.ard_adamw_values(50, (ard.CAdamWTensor * 50)(*t), outs, outs, None) == -1


# ---- the binding -----------------------------------------------------------------------------------

def test_calls_marshal_their_tensors():
    bf16 = torch.bfloat16
    with D.dry_run() as lib:
        X, w, r = fake(6, 5, 24, dtype=bf16), fake(24), fake(30)
        out = (fake(6, 5, 24, dtype=bf16), r, r)
        got = ard.layer_norm_fwd(X, w, w, out=out, stream=STREAM)
        assert got[0] is out[0] and got[1] is r and D.launches(lib)[0] == 1
        grads = ard.layer_norm_bwd(X, X, w, r, r, out=(X, w, None), ws=fake_ws(), stream=STREAM)
        assert grads[0] is X and grads[1] is w and grads[2] is None
        assert ard.layer_norm_bwd(X, X, None, r, r, out=(X, None, None), stream=STREAM)[1:] == (None, None)
        ard.layer_norm_fwd(fake(30, 24), fake(20), fake(20), D=20, out=(fake(30, 24), r, r), stream=STREAM)
        S = fake(4, 16)
        f, v, o = (strided((9, 4, 16), (192, 48, 1), bf16) for _ in range(3))
        h, ck = fake(9, 4, 16, dtype=bf16), fake(2, 4, 16)
        got = ard.glr_fwd(f, v, o, c0=fake(4, 16), lengths=fake(4, dtype=torch.int32), out=(h, S, ck), stream=STREAM)
        assert got[0] is h and got[2] is ck
        assert ard.glr_fwd(f, v, train=False, out=(h, S, None), stream=STREAM)[2] is None
        got = ard.glr_bwd(f, v, o, h, ck, out=(f, v, o, S), stream=STREAM)
        assert got[2] is o and got[3] is S
        first = [strided((4, 4, 16), (16, 64, 1), bf16) for _ in range(3)]   # batch first in memory
        got = ard.glr_bwd(first[0], first[1], None, first[2], fake(1, 4, 16), out=[fake(4, 4, 16, dtype=bf16) for _ in range(2)] + [None, S], stream=STREAM)
        assert got[2] is None
        D.launches(lib)
        p, g, m = fake(300), fake(300, dtype=bf16), fake(300)
        assert ard.adamw_step([p], [g], [m], (m,), copies=[None], stream=STREAM) is None
        c8, u8, s = fake(300, dtype=torch.int8), fake(300, dtype=torch.uint8), fake(2)
        ard.adamw_step([p] * 60, [g] * 60, [c8] * 60, [u8] * 60, [s] * 60, [s] * 60, [g] * 60, step=5, grad_scale=fake(1), stream=STREAM)
        assert D.launches(lib) == (3, ["adamw_kernel"] * 3)
        assert ard.adamw_values([c8], [u8], [s], [s], out=([p], [m]), stream=STREAM)[0][0] is p


def test_values_go_into_any_pair_of_lists():
    """A pair that is made item by item has no other owner than the call."""
    c8, u8 = fake(300, dtype=torch.int8), fake(300, dtype=torch.uint8)
    m, v = fake(300), fake(300)
    with D.dry_run() as lib:
        for out in (([m], [v]), [[m], (v,)], map(list, ((m,), (v,))), ([t] for t in (m, v)), (map(lambda t: t, [m]), iter([v]))):
            kept = out if isinstance(out, (list, tuple)) else None
            got = ard.adamw_values([c8], [u8], [fake(2)], [fake(2)], out=out, stream=STREAM)
            assert kept is None or got is kept
            if kept is None:
                junk = [[i] for i in range(100)]   # (takes the memory of lists that were let go)
                assert len(got) == 2 and got[0][0] is m and got[1][0] is v and len(junk) == 100
            assert D.launches(lib) == (1, ["adamw_values_kernel"])
        for bad in (iter([[m]]), map(list, ((m,), (v,), (m,))), 3):
            with pytest.raises((TypeError, ValueError)):
                ard.adamw_values([c8], [u8], [fake(2)], [fake(2)], out=bad, stream=STREAM)
        assert D.launches(lib)[0] == 0


def test_calls_refuse():
    bf16 = torch.bfloat16
    X, w, r, S, many = fake(30, 24, dtype=bf16), fake(24), fake(30), fake(4, 16), fake(600, 24, dtype=bf16)
    f, h, ck = fake(9, 4, 16), fake(9, 4, 16), fake(2, 4, 16)
    p, c8, u8, s = fake(300), fake(300, dtype=torch.int8), fake(300, dtype=torch.uint8), fake(2)
    kw = dict(stream=STREAM)
    with D.dry_run() as lib:
        for error, call in [
                (ValueError, lambda: ard.layer_norm_fwd(X, fake(23), out=(X, r, r), **kw)),
                (TypeError, lambda: ard.layer_norm_fwd(X, w, fake(24, dtype=bf16), out=(X, r, r), **kw)),
                (TypeError, lambda: ard.layer_norm_fwd(fake(30, 24, dtype=torch.float16), out=(X, r, r), **kw)),
                (AssertionError, lambda: ard.layer_norm_fwd(torch.zeros(3, 4), **kw)),
                (AssertionError, lambda: ard.layer_norm_fwd(strided((24, 30), (1, 24), bf16), out=(X, w, w), **kw)),
                (AssertionError, lambda: ard.layer_norm_fwd(strided((5, 5, 24), (144, 24, 1), bf16), out=(X, r, r), **kw)),
                (ValueError, lambda: ard.layer_norm_fwd(X, D=9, out=(X, r, r), **kw)),
                (ValueError, lambda: ard.layer_norm_fwd(X, out=(X, r), **kw)),
                (ValueError, lambda: ard.layer_norm_fwd(X, out=(X, r, fake(29)), **kw)),
                (TypeError, lambda: ard.layer_norm_fwd(X, out=(fake(30, 24), r, r), **kw)),
                (TypeError, lambda: ard.layer_norm_bwd(X, X, w, None, r, out=(X, w, w), ws=fake_ws(), **kw)),
                (ValueError, lambda: ard.layer_norm_bwd(fake(29, 24, dtype=bf16), X, w, r, r, out=(X, w, w), ws=fake_ws(), **kw)),
                (ValueError, lambda: ard.layer_norm_bwd(X, X, w, r, r, out=(X, fake(25), w), ws=fake_ws(), **kw)),
                (ard.ArdError, lambda: ard.layer_norm_bwd(many, many, w, fake(600), fake(600), out=(many, w, w), ws=fake_ws(16), **kw)),
                (ValueError, lambda: ard.glr_fwd(f, fake(8, 4, 16), out=(h, S, ck), **kw)),
                (ValueError, lambda: ard.glr_fwd(f, f, strided((9, 4, 16), (192, 48, 1)), out=(h, S, ck), **kw)),
                (TypeError, lambda: ard.glr_fwd(f, fake(9, 4, 16, dtype=bf16), out=(h, S, ck), **kw)),
                (TypeError, lambda: ard.glr_fwd(f, f, c0=fake(4, 16, dtype=bf16), out=(h, S, ck), **kw)),
                (ValueError, lambda: ard.glr_fwd(f, f, out=(h, S, fake(1, 4, 16)), **kw)),
                (ValueError, lambda: ard.glr_fwd(f, f, H=17, out=(h, S, ck), **kw)),
                (ValueError, lambda: ard.glr_fwd(f, f, out=(strided((9, 4, 16), (0, 16, 1)), S, ck), **kw)),
                (ard.ArdError, lambda: ard.glr_fwd(f, f, c0=S, out=(h, S, ck), **kw)),
                (TypeError, lambda: ard.glr_bwd(f, f, None, h, None, out=(f, f, None, S), **kw)),
                (ValueError, lambda: ard.glr_bwd(f, f, None, h, ck, out=(f, f, f, S), **kw)),
                (ValueError, lambda: ard.glr_bwd(f, f, f, h, ck, out=(f, strided((9, 4, 16), (192, 48, 1)), f, S), **kw)),
                (TypeError, lambda: ard.adamw_step([p], [p], [p], None, **kw)),
                (ValueError, lambda: ard.adamw_step([p], [p], [p], [p, p], **kw)),
                (TypeError, lambda: ard.adamw_step([p], [p], [c8], [u8], **kw)),
                (ValueError, lambda: ard.adamw_step([p], [p], [c8], [u8], [s], **kw)),
                (ValueError, lambda: ard.adamw_step([p], [p], [c8], [u8], [fake(3)], [s], **kw)),
                (TypeError, lambda: ard.adamw_step([p], [p], [p], [p], copies=[p], **kw)),
                (ValueError, lambda: ard.adamw_step([fake(299)], [p], [p], [p], **kw)),
                (TypeError, lambda: ard.adamw_step([1], [p], [p], [p], **kw)),
                (TypeError, lambda: ard.adamw_step(p, [p], 3, [p], **kw)),
                (TypeError, lambda: ard.adamw_step([p], [p], [p], [p], step=1.5, **kw)),
                (ValueError, lambda: ard.adamw_values([c8], [u8], [s], [s], out=([p],), **kw)),
                (ValueError, lambda: ard.adamw_values([c8], [u8], [s], [s], out=([p], [fake(299)]), **kw))]:
            with pytest.raises(error):
                call()
        assert D.launches(lib)[0] == 0


def test_signatures_can_be_read():
    want = dict(
        layer_norm_fwd="X, gamma=None, beta=None, eps=1e-05, D=None, out=None, stream=None", layer_norm_bwd="dY, X, gamma, mean, rstd, D=None, out=None, ws=None, stream=None",
        glr_fwd="f, v, o=None, c0=None, lengths=None, train=True, H=None, out=None, ws=None, stream=None",
        glr_bwd="f, v, o, dh, ckpt, dcT=None, lengths=None, H=None, out=None, ws=None, stream=None",
        adamw_step="params, grads, m, v, m_scale=None, v_scale=None, copies=None, lr=0.001, beta1=0.9, beta2=0.999, eps=1e-08, weight_decay=0.01, step=1, grad_scale=None, "
                   "stream=None",
        adamw_values="m, v, m_scale, v_scale, out=None, stream=None")
    for name, params in want.items():
        assert str(inspect.signature(getattr(ard, name))) == f"({params})", name


def test_states_before_the_first_step():
    params = [torch.zeros(3, 5), torch.zeros(300), torch.zeros(0)]
    s = ard.adamw_state(params)
    assert s["m_scale"] is None and [t.shape for t in s["m"]] == [p.shape for p in params] and s["v"][0].dtype == torch.float32
    s = ard.adamw_state(params, 8)
    assert s["m"][0].dtype == torch.int8 and s["v"][1].dtype == torch.uint8 and [t.numel() for t in s["m_scale"]] == [1, 2, 0] and s["v"][0].shape == (3, 5)
    assert C.sizeof(ard.CAdamWTensor) == 64
    with pytest.raises(ValueError):
        ard.adamw_state(params, 4)
