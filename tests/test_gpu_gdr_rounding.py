"""The gated delta rule's bf16 results are fp32 results rounded once: how many of them are bf16's nearest to the 64-bit value."""
import numpy as np
import pytest
import torch

from oracle import gdr as L
from paper_2203_05705_amd import binding as ard
from test_gpu_gdr import _inputs
from util import from_vals, raw_bits

pytestmark = pytest.mark.gpu

# A result that is off by e before it is rounded goes to the wrong neighbour where one of bf16's borders lies between it and the exact value: in a share e / (spacing of
# bf16) of all places.  On the way to a result there are some 20 fp32 roundings of sums of its size (12 products into each sum, the chain of sums, exponentials, lengths), each
# 2^-24 / sqrt(3) as they come: sqrt(20) of them 1.5e-7, three chunks behind each other 2.7e-7.  Results of at least the tensor's rms are 2^-8 rms or more apart, so 2.7e-7 x 256 =
# 7e-5 of them, and four deviations of such a count.  (Factors of 16 bits: 3e-4 of o and dq, 6e-4 to 1e-3 of dk.)
SHARE = 7e-5


def _nearest(x):
    """Bits of the bf16 value nearest to each, ties to even, straight from 64 bits."""
    e = np.floor(np.log2(np.abs(np.where(x == 0, 1.0, x)))) - 7      # (the spacing's exponent)
    v = np.rint(x / 2.0 ** e) * 2.0 ** e
    return (v.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (128, 48), (40, 128)])
def test_bf16_results_are_rounded_once(Dk, Dv):
    T, B, Hk, H = 130, 8, 4, 4
    x, do, S0, dST = _inputs(T, B, Hk, H, Dk, Dv, "bf16", Dk + Dv)
    s = Dk ** -0.5
    ro, _, states = L.gdr_fwd(*x, S0, None, s)
    want = dict(zip(("dq", "dk", "dv"), L.gdr_bwd(*x, states, do, dST, None, s)), o=ro)
    xd, S = [from_vals(t, "bf16") for t in x], from_vals(S0, "f32")
    o, _, ckpt = ard.gdr_fwd(*xd, S0=S)
    got = dict(zip(("dq", "dk", "dv"), ard.gdr_bwd(*xd, from_vals(do, "bf16"), ckpt, dST=from_vals(dST, "f32"))), o=o)
    alone, _, _ = ard.gdr_fwd(*xd, S0=S, train=False)
    assert torch.equal(alone, o)
    shares, bounds = {}, {}
    for what, ref in want.items():
        large = np.abs(ref) >= np.sqrt(np.mean(ref * ref))
        shares[what] = float(np.mean((raw_bits(got[what].contiguous()) != _nearest(ref))[large]))
        bounds[what] = SHARE + 4 * np.sqrt(SHARE / large.sum())
    assert all(shares[what] <= bounds[what] for what in want), (shares, bounds)
