"""Trains a small decoder with this library alone, and writes text with it: every product with an INT8 weight, attention, rotary positions, norms, the loss
and all of their gradients are its kernels, the INT8 weights are updated by its optimizer step, and tokens are generated over its paged cache.

    python -m paper_2407_08296_amd.example_decoder_lm [--steps N] [--layers N] [--generate N]

The text is packed sequences of all lengths in which a run of tokens repeats itself, so that a token is known from what stood a period before it: what
attention is for.  A block is

    h <- h + gate_1 * norm(W_o attention(rope(W_q u), rope(W_k u), W_v u)),   u = norm(h)
    h <- h + gate_2 * norm(W_down(silu(W_gate u) * W_up u)),                  u = norm(h)

with learned gates per channel and two query heads on each key head.  torch holds memory, draws the text, and runs Adam on what is not an INT8 matrix.
"""
from __future__ import annotations

import argparse

import torch

from . import qgalore as qg
from .example_ffn_lm import Int8Matrix

VOCAB, HIDDEN, FFN, HEADS, KEY_HEADS, D = 512, 256, 688, 8, 4, 32
SCALE, EPS, PAGE = 1.0, 1e-6, 16
DEV = "cuda"
QKV = (HEADS + 2 * KEY_HEADS) * D


def split(x: torch.Tensor):
    """q, k and v of a layer's output [tokens][QKV], as views."""
    T = x.shape[0]
    return (x[:, :HEADS * D].view(T, HEADS, D), x[:, HEADS * D:(HEADS + KEY_HEADS) * D].view(T, KEY_HEADS, D),
            x[:, (HEADS + KEY_HEADS) * D:].view(T, KEY_HEADS, D))


class Model:
    def __init__(self, layers: int, seed: int = 0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        matrix = lambda m, n, i, k: Int8Matrix(m, n, n ** -0.5, 100 * i + k, gen)
        self.blocks = [(matrix(QKV, HIDDEN, i, 0), matrix(HIDDEN, HEADS * D, i, 1), matrix(FFN, HIDDEN, i, 2), matrix(FFN, HIDDEN, i, 3),
                        matrix(HIDDEN, FFN, i, 4)) for i in range(layers)]
        self.freqs = qg.rope_frequencies(D)
        self.embed = torch.randn(VOCAB, HIDDEN, device=DEV, generator=gen)
        self.head = torch.randn(VOCAB, HIDDEN, device=DEV, generator=gen) * 0.02
        ones = lambda n: [torch.ones(HIDDEN, device=DEV) for _ in range(n)]
        self.w_pre, self.w_post = ones(2 * layers + 1), ones(2 * layers)      # ahead of and behind each half block
        self.gates = [torch.full((HIDDEN,), 0.5, device=DEV) for _ in range(2 * layers)]
        self.dense = [self.embed, self.head, *self.w_pre, *self.w_post, *self.gates]
        self.adam = torch.optim.Adam(self.dense, lr=3e-3)

    def _add(self, h, y, half):
        """The stream behind half a block, and the next half's input."""
        return qg.residual_norm_forward(h, y, self.w_post[half], self.gates[half], self.w_pre[half + 1], SCALE, EPS)

    def loss_and_gradients(self, tokens, labels, cu, positions):
        """Mean loss of the labels inside the vocabulary; gradients of the INT8 weights (returned) and of self.dense (.grad).  cu: boundaries of the
        packed sequences, positions: of each token in its own."""
        h = self.embed[tokens]                                        # the residual stream, fp32
        _, u = qg.residual_norm_forward(h, w_pre=self.w_pre[0], eps=EPS)
        kept = []
        for i, (wqkv, wo, wg, wu, wd) in enumerate(self.blocks):
            x = u
            qkv, _ = qg.int8_linear_act_forward(x, *wqkv.weight())
            q, k, v = split(qkv)
            qg.rope_forward(q, k, positions, self.freqs, out=(q, k))
            a, lse = qg.attention_forward(q, k, v, cu)
            y, _ = qg.int8_linear_act_forward(a.view(-1, HEADS * D), *wo.weight())
            h, u = self._add(h, y, 2 * i)
            b, zg, zu = qg.int8_gated_forward(u, *wg.weight(), *wu.weight(), want_z=True)
            z, _ = qg.int8_linear_act_forward(b, *wd.weight())
            kept.append((x, qkv, a, lse, y, h, u, zg, zu, b, z))
            h, u = self._add(h, z, 2 * i + 1)
            kept[-1] += (h,)
        head = self.head.bfloat16()
        loss, lse = qg.head_loss_forward(u, head, labels)
        learned = (labels >= 0) & (labels < VOCAB)
        count = learned.sum().clamp(min=1)
        du, dhead = qg.head_loss_backward(u, head, labels, lse, learned / count)
        n = len(self.blocks)
        grads, dh = [], None
        dpre, dpost, dgates = [None] * (2 * n + 1), [None] * (2 * n), [None] * (2 * n)

        def back(du, dh, h_next, y, half):
            dh, dy, dpre[half + 1], dpost[half], dgates[half] = qg.residual_norm_backward(
                du, dh, h_next, y, self.w_post[half], self.gates[half], self.w_pre[half + 1], SCALE, EPS)
            return dh, dy
        for i in reversed(range(n)):
            wqkv, wo, wg, wu, wd = self.blocks[i]
            x, qkv, a, lse, y, h_mid, u, zg, zu, b, z, h_end = kept[i]
            dh, dz = back(du, dh, h_end, z, 2 * i + 1)
            db, Gd, _ = qg.int8_linear_act_backward(dz, None, b, *wd.weight())
            du, Gg, Gu = qg.int8_gated_backward(db, zg, zu, u, *wg.weight(), *wu.weight())
            dh, dy = back(du, dh, h_mid, y, 2 * i)
            da, Go, _ = qg.int8_linear_act_backward(dy, None, a.view(-1, HEADS * D), *wo.weight())
            q, k, v = split(qkv)
            dqkv = torch.empty_like(qkv)
            dq, dk, dv = split(dqkv)
            qg.attention_backward(da.view(-1, HEADS, D), q, k, v, a, lse, cu, out=(dq, dk, dv))
            qg.rope_backward(dq, dk, positions, self.freqs, out=(dq, dk))
            du, Gqkv, _ = qg.int8_linear_act_backward(dqkv, None, x, *wqkv.weight())
            grads.insert(0, (Gqkv, Go, Gg, Gu, Gd))
        dh, _, dpre[0], _, _ = qg.residual_norm_backward(du, dh, self.embed[tokens], w_pre=self.w_pre[0], eps=EPS)
        order = torch.argsort(tokens, stable=True)                    # sums per token in a fixed order
        ends = torch.bincount(tokens, minlength=VOCAB).cumsum(0)
        sums = torch.cat([torch.zeros(1, HIDDEN, dtype=torch.float64, device=DEV), dh[order].double().cumsum(0)])
        dembed = (sums[ends] - sums[torch.cat([ends.new_zeros(1), ends[:-1]])]).float()
        for p, g in zip(self.dense, [dembed, dhead.float(), *dpre, *dpost, *dgates]):
            p.grad = g
        return loss.sum() / count, grads

    def train_step(self, batch, step: int, hp: qg.HParams) -> torch.Tensor:
        loss, grads = self.loss_and_gradients(*batch)
        for block, gs in zip(self.blocks, grads):
            for w, G in zip(block, gs):
                w.update(G, step, hp)
        self.adam.step()
        return loss

    def generate(self, prompts: torch.Tensor, new: int) -> torch.Tensor:
        """The likeliest `new` tokens behind each row of prompts [sequences][length], one at a time over a paged cache."""
        B, length = prompts.shape
        width = -(-(length + new) // PAGE)
        table = torch.randperm(B * width, device=DEV).to(torch.int32).view(B, width)
        caches = [[torch.empty(B * width, PAGE, KEY_HEADS, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for _ in self.blocks]
        sequence = torch.arange(B, dtype=torch.int32, device=DEV)
        head = self.head.bfloat16().float()

        def run(tokens, sequence, positions, attend):
            """The logits' inputs of tokens at their positions, whose keys and values enter the cache."""
            h = self.embed[tokens]
            _, u = qg.residual_norm_forward(h, w_pre=self.w_pre[0], eps=EPS)
            for i, (wqkv, wo, wg, wu, wd) in enumerate(self.blocks):
                qkv, _ = qg.int8_linear_act_forward(u, *wqkv.weight())
                q, k, v = split(qkv)
                q = qg.cache_append(q, k, v, positions, *caches[i], table, sequence=sequence, freqs=self.freqs)
                a = attend(q, k, v, positions, caches[i])
                y, _ = qg.int8_linear_act_forward(a.view(-1, HEADS * D), *wo.weight())
                h, u = self._add(h, y, 2 * i)
                z, _ = qg.int8_linear_act_forward(qg.int8_gated_forward(u, *wg.weight(), *wu.weight())[0], *wd.weight())
                h, u = self._add(h, z, 2 * i + 1)
            return u

        def whole(q, k, v, positions, cache):        # the prompt: attention over itself, its keys turned as the cache's are
            k, _ = qg.rope_forward(k, None, positions, self.freqs)
            cu = torch.arange(0, B * length + 1, length, dtype=torch.int32, device=DEV)
            return qg.attention_forward(q, k, v, cu)[0]
        u = run(prompts.flatten(), sequence.repeat_interleave(length), torch.arange(length, device=DEV).repeat(B), whole).view(B, length, HIDDEN)[:, -1]
        out = []
        for t in range(length, length + new):
            out.append((u.float() @ head.t()).argmax(1))
            if t + 1 < length + new:
                lengths = torch.full((B,), t + 1, dtype=torch.int32, device=DEV)
                u = run(out[-1], sequence, torch.full((B,), t, device=DEV), lambda q, k, v, positions, cache: qg.attention_paged(q, *cache, table, lengths))
        return torch.stack(out, 1)


def periodic(gen: torch.Generator, lengths, padding: int = 0):
    """A batch (tokens, labels, cu, positions): packed sequences, each a random run of 8 to 24 tokens over and over; behind them padding that is not learned."""
    tokens, labels, positions = [], [], []
    for n in lengths:
        period = int(torch.randint(8, 25, (1,), device=DEV, generator=gen))
        run = torch.randint(0, VOCAB, (period,), device=DEV, generator=gen).repeat(-(-(n + 1) // period))[:n + 1]
        known = torch.arange(1, n + 1, device=DEV) >= period          # the first run cannot be known
        tokens.append(run[:-1])
        labels.append(torch.where(known, run[1:], -100))
        positions.append(torch.arange(n, device=DEV))
    end = torch.zeros(padding, dtype=torch.int64, device=DEV)
    cu = torch.tensor([0] + list(lengths)).cumsum(0).to(torch.int32).to(DEV)
    return torch.cat(tokens + [end]), torch.cat(labels + [end - 100]), cu, torch.cat(positions + [end])


def train(steps: int, layers: int = 2, seed: int = 0, report=None):
    """Trains for `steps` steps; returns the model and the losses."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    model = Model(layers, seed)
    hp = qg.hparams(lr=4e-3, alpha=0.25)
    losses = []
    for step in range(1, steps + 1):
        lengths = torch.randint(40, 200, (16,), device=DEV, generator=gen).tolist()
        losses.append(model.train_step(periodic(gen, lengths, padding=-sum(lengths) % 64), step, hp))
        if report is not None and (step == 1 or step % 20 == 0):
            report(f"step {step}: loss {float(losses[-1]):.3f}")
    return model, [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--generate", type=int, default=24)
    a = ap.parse_args()
    model, _ = train(a.steps, a.layers, report=lambda s: print(s, flush=True))
    tokens, _, _, _ = periodic(torch.Generator(device=DEV).manual_seed(1), [60])
    print("prompt ", tokens[-30:].tolist(), "\nwritten", model.generate(tokens[None], a.generate)[0].tolist())
