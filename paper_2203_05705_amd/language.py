"""A small recurrent language model that learns from a teacher's largest logits, trained with this library alone:

    x = embedding of the tokens;  for each block  n = layer norm(x);  q, k, v, f, b = one product of n;
    o = gated delta rule of them;  x = x + a product of o;
    logits = layer norm(x) times the embedding table;  loss against the teacher's logits and the labels

forward and backward, one AdamW step over all of its tensors, and generation from a state of fixed size.
``python -m paper_2203_05705_amd.language`` trains one on sequences of a random chain of tokens, whose true
probabilities are the teacher.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as ard


class Model:
    """V tokens, D-wide residual stream, blocks of H heads with states of Dk x Dv whose queries and keys Hk heads give.  Masters are
    fp32; in bf16 everything reads bf16 copies that the optimizer's step writes."""

    def __init__(self, V: int, D: int, blocks: int = 2, H: int = 4, Hk: int | None = None, Dk: int = 32, Dv: int = 32, dtype=torch.bfloat16, bits: int = 32,
                 seed: int = 0, device="cuda"):
        gen = torch.Generator(device="cpu").manual_seed(seed)
        self.V, self.D, self.H, self.Hk, self.Dk, self.Dv, self.dtype = V, D, H, Hk or H, Dk, Dv, dtype
        self.parts = [self.Hk * Dk, self.Hk * Dk, H * Dv, H, H]      # of a block's product: q, k, v, f, b

        def uniform(rows, cols, scale=1.0):
            return ((torch.rand((rows, cols), generator=gen) * 2 - 1) * (scale * (6.0 / (rows + cols)) ** 0.5)).to(device)
        # the table, which is the logits' weight too; of each block gamma, beta, W, Wy; the last norm's gamma and beta
        self.params = [(torch.randn((V, D), generator=gen) * D ** -0.5).to(device)]
        for _ in range(blocks):
            self.params += [torch.ones(D, device=device), torch.zeros(D, device=device), uniform(sum(self.parts), D), uniform(D, H * Dv, 0.5)]
        self.params += [torch.ones(D, device=device), torch.zeros(D, device=device)]
        self.copies = None if dtype == torch.float32 else [p.to(dtype) for p in self.params]
        self.state = ard.adamw_state(self.params, bits)
        self.steps = 0

    def weights(self):
        """(table, blocks of (gamma, beta, W, Wy), last gamma, last beta)"""
        w = self.copies or self.params
        return w[0], [w[i:i + 4] for i in range(1, len(w) - 2, 4)], w[-2], w[-1]

    def _parts(self, z, T, B):
        """q, k, v, f, b as they lie in the rows of a block's product."""
        q, k, v, f, b = z.view(T, B, -1).split(self.parts, dim=-1)
        return q.unflatten(-1, (self.Hk, self.Dk)), k.unflatten(-1, (self.Hk, self.Dk)), v.unflatten(-1, (self.H, self.Dv)), f, b

    def empty_state(self, B):
        """The states of all blocks before the first token of B sequences."""
        return [torch.zeros((B, self.H, self.Dk, self.Dv), device=self.params[0].device) for _ in self.weights()[1]]

    def forward(self, ids, S0=None, lengths=None):
        """int32 tokens ids [T, B] (outside 0 .. V-1: padding) -> (logits [T * B, V], states, what backward() needs)"""
        T, B = ids.shape
        E, blocks, gamma, beta = self.weights()
        x = ard.embed_fwd(ids, E, scale=self.D ** 0.5).view(T * B, self.D)
        states, saved = [], []
        for i, (g, c, W, Wy) in enumerate(blocks):
            n, mean, rstd = ard.layer_norm_fwd(x, g, c)
            z = ard.drop_gemm_fwd(n, W)
            o, S, ckpt = ard.gdr_fwd(*self._parts(z, T, B), S0=None if S0 is None else S0[i], lengths=lengths)
            saved.append((x, n, mean, rstd, z, o, ckpt))
            x = x + ard.drop_gemm_fwd(o.view(T * B, -1), Wy)
            states.append(S)
        n, mean, rstd = ard.layer_norm_fwd(x, gamma, beta)
        return ard.drop_gemm_fwd(n, E), states, (ids, lengths, saved, x, n, mean, rstd)

    def backward(self, saved, dlogits, dS=None):
        """(gradients in the order of params, gradients of the states before the first token)"""
        ids, lengths, blocks_saved, x, n, mean, rstd = saved
        T, B = ids.shape
        E, blocks, gamma, beta = self.weights()
        dE = ard.drop_gemm_bwd_weight(dlogits, n)
        dx, dgamma, dbeta = ard.layer_norm_bwd(ard.drop_gemm_bwd_data(dlogits, E), x, gamma, mean, rstd)
        grads, dS0 = [dgamma, dbeta], [None] * len(blocks)
        for i in reversed(range(len(blocks))):
            g, _, W, Wy = blocks[i]
            x, n, mean, rstd, z, o, ckpt = blocks_saved[i]
            dWy = ard.drop_gemm_bwd_weight(dx, o.view(T * B, -1))
            do = ard.drop_gemm_bwd_data(dx, Wy).view(o.shape)
            dz = torch.empty_like(z)
            dS0[i] = ard.gdr_bwd(*self._parts(z, T, B), do, ckpt, dST=None if dS is None else dS[i], lengths=lengths, out=(*self._parts(dz, T, B), None))[5]
            dW = ard.drop_gemm_bwd_weight(dz, n)
            d, dg, db = ard.layer_norm_bwd(ard.drop_gemm_bwd_data(dz, W), x, g, mean, rstd)
            dx = d.add_(dx)
            grads = [dg, db, dW, dWy] + grads
        # the table's second share, added where the logits' product left the first
        ard.embed_bwd(ids, dx.view(T, B, self.D), self.V, scale=self.D ** 0.5, beta=1.0, out=dE)
        return [dE] + grads, dS0

    def learn(self, ids, top_ids, top, labels, temperature=2.0, alpha=0.7, lengths=None, lr=1e-3):
        """One step on tokens ids [T, B] with the teacher's logits top of the tokens top_ids [T * B, K] and labels [T * B]
        -> losses [T * B], of which the mean is brought down"""
        logits, _, saved = self.forward(ids, lengths=lengths)
        weight = torch.full((logits.shape[0],), 1.0 / logits.shape[0], device=logits.device)
        loss, _, dlogits = ard.distill_fwd(logits, top_ids, top, labels=labels, temperature=temperature, alpha=alpha, dloss=weight,
                                           out=(None, None, logits))       # the gradient takes the logits' place
        self.update(self.backward(saved, dlogits)[0], lr=lr)
        return loss

    def update(self, grads, lr=1e-3, weight_decay=0.01):
        """One AdamW step over all tensors."""
        self.steps += 1
        s = self.state
        ard.adamw_step(self.params, grads, s["m"], s["v"], s["m_scale"], s["v_scale"], self.copies, lr=lr, weight_decay=weight_decay, step=self.steps)

    def step(self, ids, states):
        """Generation: the next logits [B, V] behind one token each, ids [B]; the states are updated in place."""
        E, blocks, gamma, beta = self.weights()
        x = ard.embed_fwd(ids, E, scale=self.D ** 0.5)
        for (g, c, W, Wy), S in zip(blocks, states):
            z = ard.drop_gemm_fwd(ard.layer_norm_fwd(x, g, c)[0], W)
            o = ard.gdr_fwd(*self._parts(z, 1, ids.numel()), S0=S, train=False, out=(None, S, None))[0]
            x = x + ard.drop_gemm_fwd(o.view(ids.numel(), -1), Wy)
        return ard.drop_gemm_fwd(ard.layer_norm_fwd(x, gamma, beta)[0], E)


def chain(V, K, gen):
    """A random chain: from each of V tokens to K others, (their ids [V, K] int32, their logits [V, K])."""
    ids = torch.rand((V, V), generator=gen, device="cuda").topk(K, dim=1).indices.int()
    return ids, 2.0 * torch.randn((V, K), generator=gen, device="cuda")


def train(iterations=200, T=64, B=32, V=500, D=128, K=8, dtype=torch.bfloat16, bits=32, lr=2e-3, seed=0, report=None):
    """Mean losses of a model that learns a chain from its sequences and its logits."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    succ, logits = chain(V, K, gen)
    share = torch.softmax(logits, dim=1)
    model, losses = Model(V, D, dtype=dtype, bits=bits, seed=seed), []
    for it in range(iterations):
        tokens = [torch.randint(V, (B,), generator=gen, device="cuda", dtype=torch.int32)]
        for _ in range(T):
            to = torch.multinomial(share[tokens[-1].long()], 1, generator=gen)
            tokens.append(succ[tokens[-1].long()].gather(1, to)[:, 0])
        tokens = torch.stack(tokens)
        at = tokens[:-1].reshape(-1).long()
        loss = model.learn(tokens[:-1], succ[at], logits[at].to(dtype), tokens[1:].reshape(-1).contiguous(), lr=lr)
        losses.append(loss.mean())
        if report and (it + 1) % report == 0:
            print(f"iteration {it + 1}: loss {float(torch.stack(losses[-report:]).mean()):.5f}", flush=True)
    return [float(v) for v in torch.stack(losses).cpu()]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--iterations", type=int, default=300)
    ap.add_argument("--fp32", action="store_true", help="activations and products in fp32 instead of bf16")
    a = ap.parse_args()
    for bits in (32, 8):
        print(f"optimizer states in {bits} bits")
        train(a.iterations, dtype=torch.float32 if a.fp32 else torch.bfloat16, bits=bits, report=50)
