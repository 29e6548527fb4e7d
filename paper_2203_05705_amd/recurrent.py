"""A residual block of a recurrent language model under a row pattern, trained with this library alone:

    n = layer norm(x);  f, v, o = the kept units of three dropped products of n;  h = gated linear recurrence of f, v, o;
    y = x + the dropped product of h back to the width of x

forward and backward, and one AdamW step over all of its tensors.  Between the products only the kept units exist
(compact activations), in the recurrence and its gradients too.  ``python -m paper_2203_05705_amd.recurrent`` trains
a block to follow slow averages of its input, with 32-bit and with 8-bit optimizer states.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as ard

IN, OUT = ard.IN_COMPACT, ard.OUT_COMPACT


class Block:
    """D-wide residual stream, H recurrent units.  Masters are fp32; in bf16 the products read bf16 copies that the
    optimizer's step writes.  bits: of the optimizer's states."""

    NAMES = ("gamma", "beta", "Wf", "Wv", "Wo", "Wy")

    def __init__(self, D: int, H: int, dtype=torch.bfloat16, bits: int = 32, seed: int = 0, device="cuda"):
        gen = torch.Generator(device="cpu").manual_seed(seed)
        self.D, self.H, self.dtype = D, H, dtype

        def uniform(rows, cols, scale=1.0):
            return ((torch.rand((rows, cols), generator=gen) * 2 - 1) * (scale * (6.0 / (rows + cols)) ** 0.5)).to(device)
        self.params = [torch.ones(D, device=device), torch.zeros(D, device=device), uniform(H, D), uniform(H, D), uniform(H, D), uniform(D, H, 0.1)]
        self.copies = None if dtype == torch.float32 else [p.to(dtype) for p in self.params]
        self.state = ard.adamw_state(self.params, bits)
        self.steps = 0

    def weights(self):
        return dict(zip(self.NAMES, self.copies or self.params))

    def forward(self, x, pat=None, c0=None, lengths=None):
        """x [T, B, D] -> (y [T, B, D], state [B, kept] fp32, what backward() needs).  pat: row pattern of the H units, whose
        kept ones c0 and the returned state hold (one pattern for as long as a state is carried)."""
        T, B, D = x.shape
        w, kept = self.weights(), ard.kept_count(pat, self.H)
        n, mean, rstd = ard.layer_norm_fwd(x, w["gamma"], w["beta"])
        flat = n.view(T * B, D)
        z = [ard.drop_gemm_fwd(flat, w[k], pat, flags=OUT, I=D, O=self.H).view(T, B, -1) for k in ("Wf", "Wv", "Wo")]
        h, cT, ckpt = ard.glr_fwd(*z, c0=c0, lengths=lengths, H=kept)
        y = ard.drop_gemm_fwd(h.view(T * B, -1), w["Wy"], None, pat, flags=IN, I=self.H, O=D)
        return x + y.view(T, B, D), cT, (x, pat, lengths, n, mean, rstd, z, h, ckpt, kept)

    def backward(self, saved, dy, dcT=None):
        """(dx, gradients in the order of NAMES, gradient of c0)."""
        x, pat, lengths, n, mean, rstd, z, h, ckpt, kept = saved
        T, B, D = x.shape
        w, rows = self.weights(), T * B
        flat, g, hf = n.view(rows, D), dy.reshape(rows, D), h.view(rows, -1)
        dWy = ard.drop_gemm_bwd_weight(g, hf, None, pat, flags=IN, I=self.H, O=D)
        dh = ard.drop_gemm_bwd_data(g, w["Wy"], None, pat, flags=IN, I=self.H, O=D)
        *dz, dc0 = ard.glr_bwd(*z, dh.view(T, B, -1), ckpt, dcT=dcT, lengths=lengths, H=kept)
        dz = [t.view(rows, -1) for t in dz]
        dW = [ard.drop_gemm_bwd_weight(t, flat, pat, flags=OUT, I=D, O=self.H) for t in dz]
        dn = [ard.drop_gemm_bwd_data(t, w[k], pat, flags=OUT, I=D, O=self.H) for t, k in zip(dz, ("Wf", "Wv", "Wo"))]
        dn = (dn[0] + dn[1]).add_(dn[2])
        dx, dgamma, dbeta = ard.layer_norm_bwd(dn.view(T, B, D), x, w["gamma"], mean, rstd)
        return dx.add_(dy), [dgamma, dbeta, *dW, dWy], dc0

    def update(self, grads, lr=1e-3, weight_decay=0.01, grad_scale=None):
        """One AdamW step over all tensors."""
        self.steps += 1
        s = self.state
        ard.adamw_step(self.params, grads, s["m"], s["v"], s["m_scale"], s["v_scale"], self.copies, lr=lr, weight_decay=weight_decay, step=self.steps,
                       grad_scale=grad_scale)

    def step(self, x, c, pat=None):
        """Generation: one position x [B, D] and the state [B, kept], which is updated in place -> y [B, D]."""
        w = self.weights()
        n = ard.layer_norm_fwd(x, w["gamma"], w["beta"])[0]
        z = [ard.drop_gemm_fwd(n, w[k], pat, flags=OUT, I=self.D, O=self.H)[None] for k in ("Wf", "Wv", "Wo")]
        h = ard.glr_fwd(*z, c0=c, train=False, H=ard.kept_count(pat, self.H), out=(None, c, None))[0]
        return x + ard.drop_gemm_fwd(h[0], w["Wy"], None, pat, flags=IN, I=self.H, O=self.D)


def averages(x):
    """What the example learns: averages of the input over some 4 steps, in every channel, of fp32 x [T, B, D]."""
    y, c = torch.empty_like(x), torch.zeros_like(x[0])
    for t in range(x.shape[0]):
        c = 0.75 * c + 0.25 * x[t]
        y[t] = c
    return y


def train(iterations=200, T=64, B=32, D=64, H=256, dp=1, dtype=torch.bfloat16, bits=32, lr=3e-3, seed=0, report=None):
    """Losses of a block that learns averages() from fresh noise at every iteration, under a row pattern of period dp whose kept
    units change from iteration to iteration."""
    block = Block(D, H, dtype, bits, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    losses = []
    for it in range(iterations):
        x = torch.randn((T, B, D), generator=gen, device="cuda").to(dtype)
        pat = ard.Pattern.row(dp, 1 + it % dp) if dp > 1 else None
        y, _, saved = block.forward(x, pat)
        error = y.float() - (x.float() + averages(x.float()))
        _, grads, _ = block.backward(saved, (error * (2.0 / error.numel())).to(dtype))
        block.update(grads, lr=lr)
        losses.append(error.square().mean())
        if report and (it + 1) % report == 0:
            print(f"iteration {it + 1}: loss {float(torch.stack(losses[-report:]).mean()):.5f}", flush=True)
    return [float(v) for v in torch.stack(losses).cpu()]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--iterations", type=int, default=300)
    ap.add_argument("--dp", type=int, default=2, help="period of the row pattern (1: nothing dropped)")
    ap.add_argument("--fp32", action="store_true", help="activations and products in fp32 instead of bf16")
    a = ap.parse_args()
    for bits in (32, 8):
        print(f"optimizer states in {bits} bits")
        train(a.iterations, dp=a.dp, dtype=torch.float32 if a.fp32 else torch.bfloat16, bits=bits, report=50)
