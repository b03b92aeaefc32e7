"""Performance cases of the operators around the INT8 linear layer in a training step or a forward pass: the residual
stream's norms, the linear layer with an epilogue (bias, activation, residual; gated pair), and the loss of a language
model's head.

Kinds of case
  norm_forward    one pass over the residual stream between two blocks: the block's output y is normed (w_post), gated,
                  scaled and added to the stream, and the sum is normed (w_pre) for the next block
                      n = w_post * y / rms(y);  h' = h + scale * gate * n;  u = w_pre * h' / rms(h')
  norm_backward   its gradients, from du and the stream's own gradient dh'
  act_forward     z = x W^T + bias, y = act(z) + residual, W an INT8 weight
  act_backward    dz = dy * act'(z), dx = dz W, G = dz^T x, dbias = the column sums of dz
  gated_forward   y = silu(x Wg^T) * (x Wu^T), two INT8 weights
  gated_backward  its gradients dx, Gg, Gu
  head_loss       cross entropy of softmax(x W^T) against labels, per token (a label outside [0, vocab): no loss)
  head_train      the same with the gradients of x and W

rms(v) = sqrt(mean(v^2) + eps).  An INT8 weight stands for W = bf16(code * scale), the values that every product of the
library multiplies with; activations and gradients are bf16, statistics, losses and the gradients of vectors fp32.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 256            # INT8 codes of a weight's row that share a scale
EPS = 1e-6
SCALE = 0.7            # of the residual branch


def listed():
    return [
        # serving: the stream of a single token, where latency is everything
        dict(name="norm_fwd_1x4096", kind="norm_forward", tokens=1, d=4096, stream="bf16", gate="none"),
        # a training batch through a mid-sized model, learned gate per channel
        dict(name="norm_fwd_4096x2048", kind="norm_forward", tokens=4096, d=2048, stream="fp32", gate="channel"),
        # a ragged batch, rows that start unaligned, gates that are activations themselves
        dict(name="norm_bwd_1000x2047", kind="norm_backward", tokens=1000, d=2047, stream="fp32", gate="token"),
        # 32 sequences of 256 tokens through a wide model
        dict(name="norm_bwd_8192x4096", kind="norm_backward", tokens=8192, d=4096, stream="bf16", gate="channel"),
        # the projection that ends a block of a model whose FFN width is odd: bias and residual in the epilogue
        dict(name="act_fwd_1000_5461_2048", kind="act_forward", tokens=1000, n=5461, m=2048, act="none", residual=True),
        # one sequence back through the first layer of a small model's FFN
        dict(name="act_bwd_256_768_2048", kind="act_backward", tokens=256, n=768, m=2048, act="gelu"),
        # serving: one token through the gated FFN of a large model, bound by the weights' bytes
        dict(name="gated_fwd_1_4096", kind="gated_forward", tokens=1, n=4096, m=11008, train=False),
        # a training batch of 16 sequences of 256 tokens through the same
        dict(name="gated_fwd_4096_4096", kind="gated_forward", tokens=4096, n=4096, m=11008, train=True),
        # a ragged batch back through the FFN of odd width
        dict(name="gated_bwd_1000_2048", kind="gated_backward", tokens=1000, n=2048, m=5461),
        # evaluation of one sequence by a small model
        dict(name="head_loss_256_768", kind="head_loss", tokens=256, h=768, vocab=32000),
        # a ragged fine-tuning batch, half of it prompt that is not learned, odd vocabulary
        dict(name="head_train_1000_2048", kind="head_train", tokens=1000, h=2048, vocab=32003, ignored=0.5),
        # a training batch of the large model
        dict(name="head_train_4096_4096", kind="head_train", tokens=4096, h=4096, vocab=32000, ignored=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range; two in three are multiples of 64, the rest whatever comes (odd ones among them)."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 1 / 3 else max(64, v // 64 * 64)


def _tokens(rng, most):
    """One token to `most`: a quarter a handful (serving), the rest a batch."""
    return _log_int(rng, 1, min(64, most)) if rng.random() < 1 / 4 else _log_int(rng, min(64, most), most)


def draw(rng):
    kind = rng.choice(["norm_forward", "norm_backward", "act_forward", "act_backward", "gated_forward", "gated_backward",
                       "head_loss", "head_train"])
    if kind.startswith("norm"):
        return dict(kind=kind, tokens=_tokens(rng, 8192), d=_size(rng, 512, 4096), stream=rng.choice(["bf16", "fp32"]),
                    gate=rng.choice(["none", "channel", "token"]))
    n = _size(rng, 512, 4096)
    if kind.startswith("head"):
        c = dict(kind=kind, tokens=_tokens(rng, 4096), h=n, vocab=_size(rng, 4000, 32000))
        if kind == "head_train":
            c["ignored"] = rng.choice([0.0, 0.1, 0.5])
        return c
    m = _size(rng, 2 * n, 11008 * n // 4096)
    if kind.startswith("act") and rng.random() < 1 / 2:
        n, m = m, n
    c = dict(kind=kind, tokens=_tokens(rng, 4096), n=n, m=m)
    if kind == "gated_forward":
        c["train"] = rng.random() < 1 / 2
    if kind.startswith("act"):
        c["act"] = rng.choice(["none", "relu", "silu", "gelu"])
    if kind == "act_forward":
        c["residual"] = rng.random() < 1 / 2
    return c


# ------------------------------------------------------------------------------------------------------ inputs
def _weight(m, n, gen):
    """INT8 codes [m][n] and scales [m][ceil(n / 256)] of N(0, 0.02) weights, scale = absmax / 127 per block of a row."""
    w = torch.randn(m, n, device=DEV, generator=gen) * 0.02
    blocks = torch.nn.functional.pad(w, (0, -n % GROUP)).view(m, -1, GROUP)
    absmax = blocks.abs().amax(2)
    codes = (blocks * (127 / absmax.clamp(min=1e-30))[:, :, None]).round().clamp(-128, 127).to(torch.int8)
    return codes.view(m, -1)[:, :n].contiguous(), absmax / 127


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    c, kind, T = case, case["kind"], case["tokens"]

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, device=DEV, generator=gen) * std + mean).to(dtype)

    s = dict(case=dict(case))
    if kind.startswith("norm"):
        d, stream = c["d"], torch.float32 if c["stream"] == "fp32" else torch.bfloat16
        s["y"] = normal(T, d, std=0.5)
        s["w_post"], s["w_pre"] = (normal(d, std=0.1, mean=1.0, dtype=torch.float32) for _ in range(2))
        s["gate"] = {"none": None, "channel": normal(d, std=0.2, mean=0.5, dtype=torch.float32),
                     "token": normal(T, d, std=0.2, mean=0.5)}[c["gate"]]
        s["h"] = normal(T, d, std=2.0, dtype=stream)      # the stream before (forward) or behind (backward) the addition
        if kind == "norm_backward":
            s["du"], s["dh"] = normal(T, d, std=1e-3), normal(T, d, std=1e-3, dtype=stream)
    elif kind.startswith("head"):
        s["x"], s["W"] = normal(T, c["h"]), normal(c["vocab"], c["h"], std=0.02)
        s["labels"] = torch.randint(0, c["vocab"], (T,), device=DEV, generator=gen)
        if kind == "head_train":
            ignored = torch.rand(T, device=DEV, generator=gen) < c["ignored"]
            s["labels"][ignored] = -100
            s["dloss"] = torch.full((T,), 1.0 / T, device=DEV)
    else:
        m, n = c["m"], c["n"]
        s["x"] = normal(T, n)
        s["W"] = _weight(m, n, gen)
        if kind.startswith("gated"):
            s["Wu"] = _weight(m, n, gen)
        if kind == "act_forward":
            s["bias"] = normal(m, std=0.1)
            s["residual"] = normal(T, m) if c["residual"] else None
        if kind.endswith("backward"):
            s["dy"], s["z"] = normal(T, m, std=1e-3), normal(T, m)
            if kind == "gated_backward":
                s["zu"] = normal(T, m)
    return s


# -------------------------------------------------------------------------------------------------- plain forms
def _dequant(weight):
    codes, scales = weight
    w = codes.float() * scales.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return w.to(torch.bfloat16).float()


def _act(z, act):
    """act(z) and act'(z)."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _norm_forward(s):
    y, h = s["y"].float(), s["h"].float()
    n = s["w_post"] * y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    gate = 1.0 if s["gate"] is None else s["gate"].float()
    h = h + SCALE * gate * n
    u = s["w_pre"] * h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    return dict(h=h.to(s["h"].dtype), u=u.to(torch.bfloat16))


def _norm_backward(s):
    y, h, du, w_pre, w_post = s["y"].float(), s["h"].float(), s["du"].float(), s["w_pre"], s["w_post"]
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    a = w_pre * du
    dh = s["dh"].float() + r * (a - h * (r * r * (a * h).mean(1, keepdim=True)))
    q = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    gate = 1.0 if s["gate"] is None else s["gate"].float()
    dn = SCALE * gate * dh
    b = w_post * dn
    dy = q * (b - y * (q * q * (b * y).mean(1, keepdim=True)))
    out = dict(dh=dh.to(s["h"].dtype), dy=dy.to(torch.bfloat16), dw_pre=(du * h * r).sum(0), dw_post=(dn * y * q).sum(0))
    if s["gate"] is not None:
        dgate = SCALE * dh * (w_post * y * q)
        out["dgate"] = dgate.sum(0) if s["gate"].dim() == 1 else dgate.to(torch.bfloat16)
    return out


def _act_forward(s):
    z = s["x"].float() @ _dequant(s["W"]).t() + s["bias"].float()
    y = _act(z, s["case"]["act"])[0]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(torch.bfloat16), z=z.to(torch.bfloat16))


def _act_backward(s):
    dz = s["dy"].float() * _act(s["z"].float(), s["case"]["act"])[1]
    return dict(dx=(dz @ _dequant(s["W"])).to(torch.bfloat16), G=(dz.t() @ s["x"].float()).to(torch.bfloat16), dbias=dz.sum(0))


def _gated_forward(s):
    x = s["x"].float()
    zg, zu = x @ _dequant(s["W"]).t(), x @ _dequant(s["Wu"]).t()
    out = dict(y=(_act(zg, "silu")[0] * zu).to(torch.bfloat16))
    if s["case"]["train"]:
        out.update(zg=zg.to(torch.bfloat16), zu=zu.to(torch.bfloat16))
    return out


def _gated_backward(s):
    x, dy, zu = s["x"].float(), s["dy"].float(), s["zu"].float()
    a, da = _act(s["z"].float(), "silu")
    dzg, dzu = dy * zu * da, dy * a
    dx = dzg @ _dequant(s["W"]) + dzu @ _dequant(s["Wu"])
    return dict(dx=dx.to(torch.bfloat16), Gg=(dzg.t() @ x).to(torch.bfloat16), Gu=(dzu.t() @ x).to(torch.bfloat16))


def _head(s):
    x, W, labels = s["x"].float(), s["W"].float(), s["labels"]
    logits = x @ W.t()
    top = logits.amax(1, keepdim=True)
    lse = (logits - top).exp().sum(1, keepdim=True).log() + top
    learned = ((labels >= 0) & (labels < W.shape[0]))[:, None]
    at = labels[:, None].clamp(0, W.shape[0] - 1)
    loss = torch.where(learned, lse - logits.gather(1, at), 0)[:, 0]
    if s["case"]["kind"] == "head_loss":
        return dict(loss=loss)
    dl = (logits - lse).exp()
    dl.scatter_add_(1, at, dl.new_full(at.shape, -1))
    dl = torch.where(learned, dl * s["dloss"][:, None], 0)
    return dict(loss=loss, dx=(dl @ W).to(torch.bfloat16), dW=(dl.t() @ x).to(torch.bfloat16))


_PLAIN = dict(norm_forward=_norm_forward, norm_backward=_norm_backward, act_forward=_act_forward, act_backward=_act_backward,
              gated_forward=_gated_forward, gated_backward=_gated_backward, head_loss=_head, head_train=_head)


# ------------------------------------------------------------------------------------------------ the library's
def _run_own(s):
    from paper_2407_08296_amd import qgalore as qg
    c, kind = s["case"], s["case"]["kind"]
    if kind == "norm_forward":
        h, u = qg.residual_norm_forward(s["h"], s["y"], s["w_post"], s["gate"], s["w_pre"], scale=SCALE, eps=EPS)
        return dict(h=h, u=u)
    if kind == "norm_backward":
        dh, dy, dw_pre, dw_post, dgate = qg.residual_norm_backward(s["du"], s["dh"], s["h"], s["y"], s["w_post"], s["gate"],
                                                                   s["w_pre"], scale=SCALE, eps=EPS)
        out = dict(dh=dh, dy=dy, dw_pre=dw_pre, dw_post=dw_post)
        return out if dgate is None else dict(out, dgate=dgate)
    if kind == "act_forward":
        y, z = qg.int8_linear_act_forward(s["x"], *s["W"], bias=s["bias"], residual=s["residual"], act=c["act"], want_z=True)
        return dict(y=y, z=z)
    if kind == "act_backward":
        dx, G, dbias = qg.int8_linear_act_backward(s["dy"], s["z"], s["x"], *s["W"], act=c["act"], want_dbias=True)
        return dict(dx=dx, G=G, dbias=dbias)
    if kind == "gated_forward":
        y, zg, zu = qg.int8_gated_forward(s["x"], *s["W"], *s["Wu"], act="silu", want_z=c["train"])
        return dict(y=y, zg=zg, zu=zu) if c["train"] else dict(y=y)
    if kind == "gated_backward":
        dx, Gg, Gu = qg.int8_gated_backward(s["dy"], s["z"], s["zu"], s["x"], *s["W"], *s["Wu"], act="silu")
        return dict(dx=dx, Gg=Gg, Gu=Gu)
    loss, lse = qg.head_loss_forward(s["x"], s["W"], s["labels"])
    if kind == "head_loss":
        return dict(loss=loss)
    dx, dW = qg.head_loss_backward(s["x"], s["W"], s["labels"], lse, s["dloss"])
    return dict(loss=loss, dx=dx, dW=dW)


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------------- bounds
def work(case):
    c, kind, T = case, case["kind"], case["tokens"]
    if kind.startswith("norm"):
        d, stream = c["d"], 4 if c["stream"] == "fp32" else 2
        gate = {"none": 0, "channel": 4 * d, "token": 2 * T * d}[c["gate"]]
        vectors = 8 * d
        if kind == "norm_forward":     # h, y -> h', u
            return dict(bytes=T * d * (2 * stream + 4) + gate + vectors, flops=12 * T * d)
        return dict(bytes=T * d * (3 * stream + 6) + 2 * (gate + vectors), flops=30 * T * d)    # du, dh', h', y -> dh, dy
    if kind.startswith("head"):
        h, V = c["h"], c["vocab"]
        learned = 1 - c.get("ignored", 0.0)
        if kind == "head_loss":
            return dict(bytes=2 * (T + V) * h + 12 * T, flops=2 * T * V * h)
        return dict(bytes=4 * (T + V) * h + 16 * T, flops=6 * T * V * h * learned)
    m, n = c["m"], c["n"]
    weight = m * n + 4 * m * -(-n // GROUP)
    if kind == "act_forward":
        return dict(bytes=2 * T * (n + 2 * m + (m if c["residual"] else 0)) + weight + 2 * m, flops=2 * T * m * n)
    if kind == "act_backward":
        z = 0 if c["act"] == "none" else 2 * T * m
        return dict(bytes=2 * T * (2 * n + m) + z + weight + 2 * m * n + 4 * m, flops=4 * T * m * n)
    if kind == "gated_forward":
        return dict(bytes=2 * T * (n + m * (3 if c["train"] else 1)) + 2 * weight, flops=4 * T * m * n)
    return dict(bytes=2 * T * (2 * n + 3 * m) + 2 * weight + 4 * m * n, flops=8 * T * m * n)


# -------------------------------------------------------------------------------------------- 64-bit definition
def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and k != "labels"}

    def weight(name):
        codes, scales = s[name]
        blocks = torch.arange(codes.shape[1], device=DEV) // GROUP
        return (codes * scales[:, blocks]).bfloat16().double()     # one fp32 product, then bf16: the weight's value

    if kind.startswith("norm"):
        def rms(v):
            return torch.sqrt(v.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS)

        gate = f.get("gate", torch.ones((), dtype=torch.float64, device=DEV))
        if kind == "norm_forward":
            h = f["h"] + SCALE * gate * (f["w_post"] * f["y"] / rms(f["y"]))
            return dict(h=h, u=f["w_pre"] * h / rms(h))
        # gradients through automatic differentiation of the formulas, in 64 bits
        leaves = {k: f[k].requires_grad_() for k in ("y", "h", "w_post", "w_pre")}
        if s["gate"] is not None:
            leaves["gate"] = gate.requires_grad_()
        u = leaves["w_pre"] * leaves["h"] / rms(leaves["h"])
        dh = f["dh"] + torch.autograd.grad(u, leaves["h"], f["du"], retain_graph=True)[0]
        dw_pre = torch.autograd.grad(u, leaves["w_pre"], f["du"])[0]
        added = SCALE * gate * (leaves["w_post"] * leaves["y"] / rms(leaves["y"]))
        to = [k for k in ("y", "w_post", "gate") if k in leaves]
        g = dict(zip(to, torch.autograd.grad(added, [leaves[k] for k in to], dh.expand_as(added))))
        out = dict(dh=dh, dy=g["y"], dw_pre=dw_pre, dw_post=g["w_post"])
        return dict(out, dgate=g["gate"]) if "gate" in g else out
    if kind.startswith("head"):
        logits = torch.matmul(f["x"], f["W"].t().contiguous())
        learned = (s["labels"] >= 0) & (s["labels"] < c["vocab"])
        logp = logits.log_softmax(1)
        del logits
        at = torch.where(learned, s["labels"], 0)
        loss = -logp[torch.arange(c["tokens"], device=DEV), at] * learned
        if kind == "head_loss":
            return dict(loss=loss)
        dl = logp.exp_()
        dl[torch.arange(c["tokens"], device=DEV), at] -= 1
        dl *= (f["dloss"] * learned)[:, None]
        return dict(loss=loss, dx=dl @ f["W"], dW=dl.t().contiguous() @ f["x"])
    act = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[c.get("act", "silu")]
    if kind == "act_forward":
        z = f["x"] @ weight("W").t().contiguous() + f["bias"]
        return dict(y=act(z) + f.get("residual", 0.0), z=z)
    if kind == "gated_forward":
        zg, zu = (f["x"] @ weight(w).t().contiguous() for w in ("W", "Wu"))
        return dict(y=act(zg) * zu, zg=zg, zu=zu) if c["train"] else dict(y=act(zg) * zu)
    z = f["z"].requires_grad_()
    if kind == "act_backward":
        dz, = torch.autograd.grad(act(z) * 1, z, f["dy"])
        return dict(dx=dz @ weight("W"), G=dz.t().contiguous() @ f["x"], dbias=dz.sum(0))
    zu = f["zu"].requires_grad_()
    dzg, dzu = torch.autograd.grad(act(z) * zu, (z, zu), f["dy"])
    return dict(dx=dzg @ weight("W") + dzu @ weight("Wu"), Gg=dzg.t().contiguous() @ f["x"], Gu=dzu.t().contiguous() @ f["x"])
