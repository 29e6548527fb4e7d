"""The gated delta rule where a workgroup makes the operands of several heads that share a key, one behind the other: all of them, or an uneven share."""
import pytest

from paper_2203_05705_amd import binding as ard
from test_gpu_gdr import _check

pytestmark = pytest.mark.gpu   # tolerances: those of test_gpu_gdr


def _shares(T, B, Hk, H):
    """Heads that each workgroup takes: one workgroup for a key head's heads from 385 (chunk, sequence, key head) on, below as many as fill 768 workgroups."""
    units, group = -(-T // ard.GDR_CHUNK) * B * Hk, H // Hk
    n = min(group, 768 // units) if units * 2 <= 768 else 1
    return [(i + 1) * group // n - i * group // n for i in range(n)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(24, 16), (72, 8)])
@pytest.mark.parametrize("T,B,Hk,H,shares,ragged", [(65, 200, 1, 3, [3], False), (65, 200, 1, 3, [3], True), (40, 193, 2, 4, [2], True), (65, 150, 1, 5, [2, 3], False),
                                                    (65, 150, 1, 5, [2, 3], True), (65, 100, 1, 7, [2, 2, 3], True), (130, 32, 2, 14, [1, 2, 2, 2], True)])
def test_heads_one_behind_the_other(T, B, Hk, H, shares, ragged, Dk, Dv, dtype):
    assert sorted(_shares(T, B, Hk, H)) == shares
    _check(T, B, Hk, H, Dk, Dv, dtype, ragged=ragged, seed=B + H)
