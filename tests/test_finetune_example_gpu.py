"""examples/finetune_step.py: the operators together, as a fine-tuning step uses them."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def plain_loss(block, w, b, table, tau, wt, wl):
    """The example's loss in 64 bits with automatic differentiation, written apart from it."""
    T, Hq, Hk, D = b["x"].shape[0], block.Hq, block.Hk, block.D
    x = b["x"].double()
    qkv = (x @ w["qkv"].T).view(T, Hq + 2 * Hk, D)
    cs = table.double()[b["pos"].long()][:, None]
    cos, sin = cs.chunk(2, -1)
    def norm_turn(y, weight):
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight
        a, c = y.chunk(2, -1)
        return torch.cat([a * cos - c * sin, c * cos + a * sin], -1)
    q, k, v = norm_turn(qkv[:, :Hq], w["q_norm"]), norm_turn(qkv[:, Hq:Hq + Hk], w["k_norm"]), qkv[:, Hq + Hk:]
    k, v = (y.repeat_interleave(Hq // Hk, 1) for y in (k, v))
    out = torch.zeros_like(q)
    for lo, hi in zip(b["cu"].tolist(), b["cu"].tolist()[1:]):
        s = torch.einsum("ihd,jhd->hij", q[lo:hi], k[lo:hi]) * D ** -0.5
        s = s.masked_fill(torch.ones(hi - lo, hi - lo, device="cuda").triu(1).bool(), -math.inf)
        out[lo:hi] = torch.einsum("hij,jhd->ihd", s.softmax(-1), v[lo:hi])
    z = (x + out.reshape(T, -1) @ w["o"].T) @ w["head"].T
    n = int(b["cu"][-1])
    ids, zt = b["ids"][:n].long(), z[:n]
    tq = (b["teacher"][:n].double() / tau).softmax(-1)
    kl = (tq * (tq.log() - (zt / tau).log_softmax(-1).gather(1, ids))).sum(1) * tau * tau
    nll = -zt.log_softmax(-1).gather(1, b["labels"][:n].long()[:, None])[:, 0]
    return (wt * kl + wl * nll).mean()


def test_gradient_of_the_block_matches_automatic_differentiation():
    import finetune_step as ex
    sd = ex.sd
    block = ex.Block(hidden=128, heads_q=4, heads_kv=2, head_dim=32, vocab=500)
    b = ex.micro_batch(block, 300, docs=3, entries=7, seed=5)
    grad = torch.zeros(block.n, dtype=torch.bfloat16, device="cuda")
    with sd.slidedp_create(0, 0) as ctx:
        loss = ex.loss_and_gradient(ctx, block, b, grad)
    w = {n: x.double().requires_grad_() for n, x in block.w.items()}
    want = plain_loss(block, w, b, ex.rotation_table(300, block.D), 2.0, 0.8, 0.2)
    assert abs(float(loss) - want.item()) < 2e-3 * want.item()       # logits are BF16: 2^-8 of each, averaged
    got = block.views(grad)
    for name, g in zip(w, torch.autograd.grad(want, list(w.values()))):
        # BF16 activations and products between some ten steps, each 2^-9 in the mean: below 2 % of the gradient's norm
        assert (got[name].double() - g).norm() < 0.02 * g.norm(), name


def test_a_few_steps_lower_the_loss():
    import finetune_step as ex
    losses = ex.train(steps=8, tokens=512, verbose=False)
    assert losses[-1] < 0.8 * losses[0] and all(a == a for a in losses)
