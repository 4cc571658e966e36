"""One decoder block fine-tuned on packed documents towards a teacher's stored top logits: the operators of
include/slidedp_ops.h produce the gradients that the step of include/slidedp.h consumes.

Per micro-batch (one per rank): projections (torch products) -> query/key norm with the rotation -> attention
within the packed documents -> output projection and vocabulary head -> distillation loss and its gradient in
one call -> the same operators' backward passes -> a flat BF16 gradient. Then once per step: the global norm over
the rank gradients, clipping, AdamW on the FP32 state and the BF16 parameters of the next step, which are the
flat buffer that the block's weights are views of.

    python examples/finetune_step.py [--steps 20] [--tokens 1536]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_34162_b200.slidedp as sd  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Block:
    """A decoder block with a vocabulary head; all weights are views of one flat BF16 buffer."""

    def __init__(self, hidden=512, heads_q=8, heads_kv=2, head_dim=64, vocab=8192, seed=0):
        self.hidden, self.Hq, self.Hk, self.D, self.vocab = hidden, heads_q, heads_kv, head_dim, vocab
        self.shapes = {"qkv": ((heads_q + 2 * heads_kv) * head_dim, hidden), "o": (hidden, heads_q * head_dim),
                       "head": (vocab, hidden), "q_norm": (head_dim,), "k_norm": (head_dim,)}
        self.n = sum(torch.Size(s).numel() for s in self.shapes.values())
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.master = torch.cat([torch.ones(s, device="cuda") if len(s) == 1 else
                                 torch.randn(s, generator=g, device="cuda").flatten() * 0.02 for s in self.shapes.values()])
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.params = self.master.to(BF16)
        self.w = self.views(self.params)

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            k = torch.Size(shape).numel()
            out[name], at = flat[at:at + k].view(shape), at + k
        return out


def rotation_table(rows, head_dim, base=10000.0):
    half = head_dim // 2
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * base ** (
        -torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return torch.cat([angle.cos(), angle.sin()], 1).to(F32)


def micro_batch(block: Block, tokens: int, docs: int, entries: int, seed: int):
    """Packed documents (a padded end among them), their positions, and what the teacher stored for each token."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cut = torch.randperm(tokens - 64, generator=g, device="cuda")[:docs].sort().values + 1
    cu = torch.cat([cut.new_zeros(1), cut]).to(torch.int32)
    t = torch.arange(tokens, device="cuda", dtype=torch.int32)
    doc = torch.searchsorted(cu, t, right=True) - 1
    ids = torch.argsort(torch.rand(tokens, block.vocab, generator=g, device="cuda"), dim=1)[:, :entries].to(torch.int32)
    ids[t >= cu[-1]] = -1                                   # padding has no teacher
    labels = torch.where(t < cu[-1], ids[:, 0], torch.full_like(t, -100))
    return dict(x=torch.randn(tokens, block.hidden, generator=g, device="cuda").to(BF16), cu=cu, pos=(t - cu[doc]).to(torch.int32),
                ids=ids.contiguous(), teacher=4.0 - 0.5 * torch.arange(entries, device="cuda", dtype=F32).repeat(tokens, 1),
                labels=labels.contiguous(), row_grad=torch.full((tokens,), 1.0 / float(cu[-1]), device="cuda"))


def loss_and_gradient(ctx: sd.Context, block: Block, b: dict, grad: torch.Tensor, temperature=2.0, w_teacher=0.8, w_label=0.2):
    """The micro-batch's mean loss; its gradient goes to ``grad`` (flat, BF16)."""
    w, g = block.w, block.views(grad)
    T, Hq, Hk, D = b["x"].shape[0], block.Hq, block.Hk, block.D
    new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    table = rotation_table(T, D)

    qkv = (b["x"] @ w["qkv"].T).view(T, Hq + 2 * Hk, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    qr, kr = new(T, Hq, D), new(T, Hk, D)
    ctx.slidedp_qk_norm_rope(q, k, w["q_norm"], w["k_norm"], table, b["pos"], qr, kr)
    out, lse = new(T, Hq, D), new(Hq, T, dtype=F32)
    ctx.slidedp_attention(qr, kr, v, out, lse, cu_docs=b["cu"])
    h = b["x"] + out.view(T, -1) @ w["o"].T
    logits = h @ w["head"].T

    loss, dist_lse = new(T, dtype=F32), new(2, T, dtype=F32)
    ctx.slidedp_distill_step(logits, b["ids"], b["teacher"], b["labels"], b["row_grad"], loss, dist_lse, logits,   # in place
                             temperature=temperature, w_teacher=w_teacher, w_label=w_label)
    g["head"].copy_(logits.T @ h)
    dh = logits @ w["head"]
    g["o"].copy_(dh.T @ out.view(T, -1))
    d_out = (dh @ w["o"]).view(T, Hq, D)
    d_qkv, dqr, dkr = new(T, Hq + 2 * Hk, D), new(T, Hq, D), new(T, Hk, D)
    ws = new(ctx.slidedp_attention_workspace(qr, kr), dtype=torch.uint8)
    ctx.slidedp_attention_backward(qr, kr, v, out, lse, d_out, dqr, dkr, d_qkv[:, Hq + Hk:], ws, cu_docs=b["cu"])
    dwq, dwk = new(D, dtype=F32), new(D, dtype=F32)
    ws = new(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8)
    ctx.slidedp_qk_norm_rope_backward(q, k, w["q_norm"], w["k_norm"], table, b["pos"], dqr, dkr, d_qkv[:, :Hq],
                                      d_qkv[:, Hq:Hq + Hk], dwq, dwk, ws)
    g["q_norm"].copy_(dwq)
    g["k_norm"].copy_(dwk)
    g["qkv"].copy_(d_qkv.view(T, -1).T @ b["x"])
    return (loss * b["row_grad"]).sum()


def train(steps=20, tokens=1536, ranks=2, lr=2e-3, verbose=True):
    block = Block()
    grads = [torch.empty(block.n, dtype=BF16, device="cuda") for _ in range(ranks)]
    batches = [micro_batch(block, tokens, docs=5, entries=16, seed=100 + r) for r in range(ranks)]
    losses = []
    with sd.slidedp_create(torch.cuda.current_device(), 0) as ctx:
        for step in range(1, steps + 1):
            loss = sum(loss_and_gradient(ctx, block, b, g) for b, g in zip(batches, grads)) / ranks
            ctx.slidedp_grad_norm(grads, block.n, 1.0 / ranks)
            norm, _ = ctx.slidedp_grad_norm_finish(1.0, fetch=True)
            ctx.slidedp_reduce_adamw_chunk(grads, block.n, block.master, block.m, block.v, block.params,
                                           sd.HParams(lr=lr, weight_decay=0.0, inv_R=1.0 / ranks, max_norm=1.0, step=step))
            losses.append(float(loss))
            if verbose:
                print(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {norm:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=1536)
    a = ap.parse_args()
    train(a.steps, a.tokens)
