"""One decoder block trained on sampled tokens with the clipped policy loss: all operators of include/slidedp_ops.h from the token ids to the
clipped gradients that the step of include/slidedp.h consumes.

Per micro-batch: token embedding -> norm -> projections (torch products) -> query/key norm with the rotation -> attention within the
packed samples -> norm, residual, norm -> feed-forward (torch) -> norm, residual, norm -> vocabulary head -> policy loss and its gradient
in one call -> the same operators' backward passes, added up in FP32. Once per step: the gradients of all tensors are clipped by
their norm into the flat BF16 gradient, then AdamW on the FP32 state and the BF16 parameters of the next step.

    python examples/policy_step.py [--steps 10] [--tokens 1024]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_34162_b200.slidedp as sd  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
CLIP = dict(clip_low=0.2, clip_high=0.28, kl_weight=0.05)


class Model:
    """Embedding, one block and a head; all weights are views of one flat BF16 buffer."""

    def __init__(self, hidden=256, heads_q=4, heads_kv=2, head_dim=64, inner=512, vocab=4096, seed=0):
        self.hidden, self.Hq, self.Hk, self.D, self.inner, self.vocab = hidden, heads_q, heads_kv, head_dim, inner, vocab
        self.shapes = {"embed": (vocab, hidden), "norm1": (hidden,), "qkv": ((heads_q + 2 * heads_kv) * head_dim, hidden), "q_norm": (head_dim,),
                       "k_norm": (head_dim,), "o": (hidden, heads_q * head_dim), "post1": (hidden,), "norm2": (hidden,),
                       "gate_up": (2 * inner, hidden), "down": (hidden, inner), "post2": (hidden,), "norm3": (hidden,), "head": (vocab, hidden)}
        self.n = sum(math.prod(s) for s in self.shapes.values())
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.master = torch.cat([torch.ones(s, device="cuda") if len(s) == 1 else torch.randn(s, generator=g, device="cuda").flatten() * 0.05
                                 for s in self.shapes.values()])
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.params = self.master.to(BF16)
        self.w = self.views(self.params)

    def views(self, flat):
        sizes = [math.prod(s) for s in self.shapes.values()]
        return {n: t.view(s) for (n, s), t in zip(self.shapes.items(), flat.split(sizes))}


def samples(model: Model, tokens: int, docs: int, seed: int):
    """Packed prompts with the tokens that were sampled after them: what is to be predicted, how likely it was then, and how good it was."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cut = torch.randperm(tokens - 32, generator=g, device="cuda")[:docs].sort().values + 1
    cu = torch.cat([cut.new_zeros(1), cut]).to(torch.int32)            # the end is padding
    t = torch.arange(tokens, device="cuda")
    doc = torch.searchsorted(cu.long(), t, right=True) - 1
    pos, length = t - cu[doc], (cu[1:] - cu[:-1])[doc.clamp(max=docs - 1)]
    ids = torch.randint(0, model.vocab, (tokens,), generator=g, device="cuda")
    labels = torch.where((pos >= length // 3) & (pos + 1 < length) & (t < cu[-1]), ids.roll(-1), -100)
    n = float((labels >= 0).sum())
    return dict(ids=torch.where(t < cu[-1], ids, -1).to(torch.int32), cu=cu, pos=pos.to(torch.int32), labels=labels.to(torch.int32),
                advantage=torch.randn(docs + 1, generator=g, device="cuda")[doc].contiguous(), row_grad=torch.full((tokens,), 1.0 / n, device="cuda"))


def rotation_table(rows, head_dim, base=10000.0):
    half = head_dim // 2
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * base ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return torch.cat([angle.cos(), angle.sin()], 1).to(F32)


def forward(ctx: sd.Context, model: Model, b: dict):
    """The logits, and what the backward pass needs."""
    w, T, Hq, Hk, D, h = model.w, len(b["ids"]), model.Hq, model.Hk, model.D, model.hidden
    new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    a = dict(table=rotation_table(T, D), x0=new(T, h), h1=new(T, h))
    ctx.slidedp_embedding(w["embed"], b["ids"], a["x0"], scale=math.sqrt(h))
    ctx.slidedp_block_norm(a["x0"], None, None, None, w["norm1"], None, a["h1"])
    a["qkv"] = (a["h1"] @ w["qkv"].T).view(T, Hq + 2 * Hk, D)
    a["q"], a["k"], a["v"] = a["qkv"][:, :Hq], a["qkv"][:, Hq:Hq + Hk], a["qkv"][:, Hq + Hk:]
    a["qr"], a["kr"], a["att"], a["lse"] = new(T, Hq, D), new(T, Hk, D), new(T, Hq, D), new(Hq, T, dtype=F32)
    ctx.slidedp_qk_norm_rope(a["q"], a["k"], w["q_norm"], w["k_norm"], a["table"], b["pos"], a["qr"], a["kr"])
    ctx.slidedp_attention(a["qr"], a["kr"], a["v"], a["att"], a["lse"], cu_docs=b["cu"])
    a["y1"] = a["att"].view(T, -1) @ w["o"].T
    a["x1"], a["h2"], a["x2"], a["h3"] = (new(T, h) for _ in range(4))
    ctx.slidedp_block_norm(a["x0"], a["y1"], w["post1"], None, w["norm2"], a["x1"], a["h2"])
    a["gu"] = a["h2"] @ w["gate_up"].T
    a["act"] = torch.nn.functional.silu(a["gu"][:, :model.inner]) * a["gu"][:, model.inner:]
    a["y2"] = a["act"] @ w["down"].T
    ctx.slidedp_block_norm(a["x1"], a["y2"], w["post2"], None, w["norm3"], a["x2"], a["h3"])
    return a["h3"] @ w["head"].T, a


def log_probabilities(ctx: sd.Context, model: Model, b: dict):
    logits, _ = forward(ctx, model, b)
    logp = torch.empty(len(b["ids"]), device="cuda")
    ctx.slidedp_policy_loss(logits, b["labels"], None, None, None, None, logp)
    return logp


def loss_and_gradient(ctx: sd.Context, model: Model, b: dict, grads: dict):
    """The micro-batch's mean loss; its gradient is added to the FP32 tensors of ``grads``."""
    w, T, Hq, Hk, D, h = model.w, len(b["ids"]), model.Hq, model.Hk, model.D, model.hidden
    new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    z, a = forward(ctx, model, b)
    loss, logp = new(T, dtype=F32), new(T, dtype=F32)
    ctx.slidedp_policy_step(z, b["labels"], b["old_logp"], b["ref_logp"], b["advantage"], b["row_grad"], loss, logp, z, **CLIP)       # in place
    dw = {n: new(*model.shapes[n], dtype=F32) for n, s in model.shapes.items() if len(s) == 1}
    ws = new(ctx.slidedp_block_norm_workspace(a["x0"]), dtype=torch.uint8)

    grads["head"] += z.T @ a["h3"]
    dx1, dy2 = new(T, h), new(T, h)
    ctx.slidedp_block_norm_backward(a["x1"], a["y2"], w["post2"], None, w["norm3"], None, z @ w["head"], dx1, dy2, None, dw["post2"], dw["norm3"], ws)
    grads["down"] += dy2.T @ a["act"]
    gate, up = a["gu"][:, :model.inner].float(), a["gu"][:, model.inner:].float()
    dact, s = (dy2 @ w["down"]).float(), torch.sigmoid(a["gu"][:, :model.inner].float())
    dgu = torch.cat([dact * up * s * (1 + gate * (1 - s)), dact * gate * s], 1).to(BF16)
    grads["gate_up"] += dgu.T @ a["h2"]
    dx0, dy1 = new(T, h), new(T, h)
    ctx.slidedp_block_norm_backward(a["x0"], a["y1"], w["post1"], None, w["norm2"], dx1, dgu @ w["gate_up"], dx0, dy1, None, dw["post1"], dw["norm2"], ws)
    grads["o"] += dy1.T @ a["att"].view(T, -1)

    d_qkv, dqr, dkr = new(T, Hq + 2 * Hk, D), new(T, Hq, D), new(T, Hk, D)
    ctx.slidedp_attention_backward(a["qr"], a["kr"], a["v"], a["att"], a["lse"], (dy1 @ w["o"]).view(T, Hq, D), dqr, dkr, d_qkv[:, Hq + Hk:],
                                   new(ctx.slidedp_attention_workspace(a["qr"], a["kr"]), dtype=torch.uint8), cu_docs=b["cu"])
    ctx.slidedp_qk_norm_rope_backward(a["q"], a["k"], w["q_norm"], w["k_norm"], a["table"], b["pos"], dqr, dkr, d_qkv[:, :Hq], d_qkv[:, Hq:Hq + Hk],
                                      dw["q_norm"], dw["k_norm"], new(ctx.slidedp_qk_norm_rope_workspace(a["q"], a["k"]), dtype=torch.uint8))
    d_qkv = d_qkv.view(T, -1)
    grads["qkv"] += d_qkv.T @ a["h1"]
    ctx.slidedp_block_norm_backward(a["x0"], None, None, None, w["norm1"], dx0, d_qkv @ w["qkv"], dx0, None, None, None, dw["norm1"], ws)
    ctx.slidedp_embedding_backward(b["ids"], dx0, grads["embed"], new(ctx.slidedp_embedding_workspace(dx0, grads["embed"]), dtype=torch.uint8),
                                   scale=math.sqrt(h), accumulate=True)
    for n, d in dw.items():
        grads[n] += d
    return (loss * b["row_grad"]).sum()


def train(steps=10, tokens=1024, micro_batches=2, lr=1e-3, verbose=True):
    model = Model()
    flat = torch.empty(model.n, dtype=BF16, device="cuda")
    clipped = list(model.views(flat).values())
    grads = {n: torch.zeros(s, device="cuda") for n, s in model.shapes.items()}
    batches = [samples(model, tokens, docs=5, seed=100 + i) for i in range(micro_batches)]
    result = torch.empty(4, dtype=torch.float64, device="cuda")
    losses = []
    with sd.slidedp_create(torch.cuda.current_device(), 0) as ctx:
        ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace(list(grads.values())), dtype=torch.uint8, device="cuda")
        for b in batches:                    # the policy that the tokens were sampled with, which is the reference too
            b["old_logp"] = b["ref_logp"] = log_probabilities(ctx, model, b)
        for step in range(1, steps + 1):
            for g in grads.values():
                g.zero_()
            loss = sum(loss_and_gradient(ctx, model, b, grads) for b in batches) / micro_batches
            ctx.slidedp_clip_grad_norm(list(grads.values()), clipped, 1.0, result, ws, scale=1.0 / micro_batches)
            ctx.slidedp_reduce_adamw_chunk([flat], model.n, model.master, model.m, model.v, model.params,
                                           sd.HParams(lr=lr, weight_decay=0.0, inv_R=1.0, max_norm=0.0, step=step))
            losses.append(float(loss))
            if verbose:
                print(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {result[1].item():.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--tokens", type=int, default=1024)
    a = ap.parse_args()
    train(a.steps, a.tokens)
