"""Trains a small feed-forward language model with this library alone: every product with an INT8 weight, every norm, the
loss and all of their gradients are its kernels, and the INT8 weights are updated by its optimizer step.

    python -m paper_2407_08296_amd.example_ffn_lm [--steps N] [--layers N]

The text is a Markov chain (each token has eight successors, so a model of single tokens can learn it: the loss falls from
log(vocab) towards the chain's entropy), and a block is

    h <- h + scale * gate * norm(W_down(silu(W_gate u) * W_up u)),   u = norm(h),

with a learned gate per channel.  torch holds memory, draws the text, and runs Adam on what is not an INT8 matrix (embedding, head,
norms and gates; a few hundred thousand numbers).
"""
from __future__ import annotations

import argparse

import torch

from . import qgalore as qg

VOCAB, HIDDEN, FFN, RANK, TOKENS = 512, 256, 688, 64, 2048
SCALE, EPS = 0.5, 1e-6
DEV = "cuda"


class Int8Matrix:
    """An m x n weight with the state of its optimizer step; the projection is refreshed every `interval` steps."""

    def __init__(self, m: int, n: int, std: float, seed: int, gen: torch.Generator, interval: int = 50):
        self.m, self.n, self.r, self.seed, self.interval = m, n, RANK, seed, interval
        self.Wq, self.Ws = qg.quant_int8(torch.randn(m, n, device=DEV, generator=gen) * std)
        q, _ = qg.orthonormalize(torch.randn(m, self.r, device=DEV, generator=gen))
        self.Pq, self.Ps = qg.quant_int4(q)
        self.M, self.V = (torch.zeros(self.r, n, device=DEV) for _ in range(2))
        self.N = torch.empty(self.r, n, dtype=torch.bfloat16, device=DEV)

    def weight(self):
        return self.Wq, self.Ws

    def update(self, G: torch.Tensor, step: int, hp: qg.HParams) -> None:
        if step % self.interval == 1:
            self.Pq, self.Ps, *_ = qg.subspace_refresh(self.Pq, self.Ps, G, self.m, self.n, self.r)
        qg.step(self.Pq, self.Ps, G, self.Wq, self.Ws, self.M, self.V, None, self.N, self.m, self.n, self.r, hp, self.seed, step)


class Model:
    def __init__(self, layers: int, seed: int = 0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.blocks = []
        for i in range(layers):
            gate_up = [Int8Matrix(FFN, HIDDEN, HIDDEN ** -0.5, 10 * i + k, gen) for k in range(2)]
            self.blocks.append((*gate_up, Int8Matrix(HIDDEN, FFN, FFN ** -0.5, 10 * i + 2, gen)))
        # what torch's Adam trains, in fp32: embedding, head, one pre-norm per block and a last one, post-norms and gates
        self.embed = torch.randn(VOCAB, HIDDEN, device=DEV, generator=gen)
        self.head = torch.randn(VOCAB, HIDDEN, device=DEV, generator=gen) * 0.02
        self.w_pre = [torch.ones(HIDDEN, device=DEV) for _ in range(layers + 1)]
        self.w_post = [torch.ones(HIDDEN, device=DEV) for _ in range(layers)]
        self.gates = [torch.full((HIDDEN,), 0.5, device=DEV) for _ in range(layers)]
        self.dense = [self.embed, self.head, *self.w_pre, *self.w_post, *self.gates]
        self.adam = torch.optim.Adam(self.dense, lr=3e-3)

    def loss_and_gradients(self, tokens: torch.Tensor, labels: torch.Tensor):
        """Mean loss of the labels inside the vocabulary; gradients of the INT8 weights (returned) and of self.dense (.grad)."""
        h = self.embed[tokens]                                        # the residual stream, fp32
        _, u = qg.residual_norm_forward(h, w_pre=self.w_pre[0], eps=EPS)
        kept = []
        for i, (wg, wu, wd) in enumerate(self.blocks):
            a, zg, zu = qg.int8_gated_forward(u, *wg.weight(), *wu.weight(), want_z=True)
            y, _ = qg.int8_linear_act_forward(a, *wd.weight())
            h, u_next = qg.residual_norm_forward(h, y, self.w_post[i], self.gates[i], self.w_pre[i + 1], SCALE, EPS)
            kept.append((u, zg, zu, a, y, h))
            u = u_next
        head = self.head.bfloat16()
        loss, lse = qg.head_loss_forward(u, head, labels)
        learned = (labels >= 0) & (labels < VOCAB)
        count = learned.sum().clamp(min=1)
        du, dhead = qg.head_loss_backward(u, head, labels, lse, learned / count)
        grads, dh = [], None
        dw_pre, dw_post, dgates = [None] * (len(self.blocks) + 1), [], []
        for i in reversed(range(len(self.blocks))):
            wg, wu, wd = self.blocks[i]
            x, zg, zu, a, y, h = kept[i]
            dh, dy, dw_pre[i + 1], dpost, dgate = qg.residual_norm_backward(du, dh, h, y, self.w_post[i], self.gates[i],
                                                                            self.w_pre[i + 1], SCALE, EPS)
            da, Gd, _ = qg.int8_linear_act_backward(dy, None, a, *wd.weight())
            du, Gg, Gu = qg.int8_gated_backward(da, zg, zu, x, *wg.weight(), *wu.weight())
            grads.insert(0, (Gg, Gu, Gd))
            dw_post.insert(0, dpost)
            dgates.insert(0, dgate)
        dh, _, dw_pre[0], _, _ = qg.residual_norm_backward(du, dh, self.embed[tokens], w_pre=self.w_pre[0], eps=EPS)
        order = torch.argsort(tokens, stable=True)                    # sums per token in a fixed order
        dembed = torch.zeros_like(self.embed)
        ends = torch.bincount(tokens, minlength=VOCAB).cumsum(0)
        sums = torch.cat([torch.zeros(1, HIDDEN, dtype=torch.float64, device=DEV), dh[order].double().cumsum(0)])
        dembed.copy_(sums[ends] - sums[torch.cat([ends.new_zeros(1), ends[:-1]])])
        for p, g in zip(self.dense, [dembed, dhead.float(), *dw_pre, *dw_post, *dgates]):
            p.grad = g
        return loss.sum() / count, grads

    def train_step(self, tokens: torch.Tensor, labels: torch.Tensor, step: int, hp: qg.HParams) -> torch.Tensor:
        loss, grads = self.loss_and_gradients(tokens, labels)
        for block, gs in zip(self.blocks, grads):
            for w, G in zip(block, gs):
                w.update(G, step, hp)
        self.adam.step()
        return loss


def chain(gen: torch.Generator, count: int, successors: torch.Tensor):
    """`count` pairs (token, next token) of the chain, one in ten without a label (as padding and prompts are)."""
    tokens = torch.randint(0, VOCAB, (count,), device=DEV, generator=gen)
    labels = successors[tokens, torch.randint(0, successors.shape[1], (count,), device=DEV, generator=gen)]
    return tokens, torch.where(torch.rand(count, device=DEV, generator=gen) < 0.1, -100, labels)


def train(steps: int, layers: int = 2, seed: int = 0, report=None):
    """Trains for `steps` steps; returns the losses."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    successors = torch.randint(0, VOCAB, (VOCAB, 8), device=DEV, generator=gen)
    model = Model(layers, seed)
    hp = qg.hparams(lr=4e-3, alpha=0.25)
    losses = []
    for step in range(1, steps + 1):
        loss = model.train_step(*chain(gen, TOKENS, successors), step, hp)
        losses.append(loss)
        if report is not None and (step == 1 or step % 20 == 0):
            report(f"step {step}: loss {float(loss):.3f}")
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    train(a.steps, a.layers, report=lambda s: print(s, flush=True))
