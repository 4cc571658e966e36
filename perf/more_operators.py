"""Measured cases of the rest of a fine-tuning step: token embedding with its gradient, the norms around a block
with its gate and residual, the clipped policy loss, and clipping by the norm over many gradient tensors.

Each case runs in two forms on the same inputs: `own` false is elementary torch arithmetic in 32
bits, rounded once at the end; `own` true calls the library. ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
_DTYPES = {"bf16": BF16, "f32": F32}


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # one token at a time: sampling from the model while it is being tuned
        dict(name="embed_forward_one_token", op="embed", train=False, T=1, V=131072, H=4096, dtype="bf16", grad="bf16", pad=0),
        # a training microbatch at the Qwen3-8B-shaped layer's width, the table's gradient beside the flat BF16 gradients
        dict(name="embed_train_8b", op="embed", train=True, T=8192, V=131072, H=4096, dtype="bf16", grad="bf16", pad=0),
        # a small model with a short vocabulary, FP32 gradient: few tokens take most of the batch, its end is padding
        dict(name="embed_train_short_vocab_f32", op="embed", train=True, T=32749, V=8000, H=1000, dtype="f32", grad="f32", pad=5),
        # one token through the end of a block and the start of the next
        dict(name="norm_forward_one_token", op="norm", train=False, T=1, H=4096, dtype="bf16", post=True, pre=True, gate="none", sig=False),
        # a training microbatch, Qwen3-8B-shaped width, norms on both sides of the block
        dict(name="norm_train_8b", op="norm", train=True, T=8192, H=4096, dtype="bf16", post=True, pre=True, gate="none", sig=False),
        # a long evaluation pass at the Qwen3-14B-shaped width, the block's output gated per token and channel
        dict(name="norm_forward_14b_gated", op="norm", train=False, T=16384, H=5120, dtype="bf16", post=False, pre=True, gate="token", sig=True),
        # a small model in FP32 with a learned gate per channel, odd sizes
        dict(name="norm_train_gate_f32", op="norm", train=True, T=1537, H=2500, dtype="f32", post=True, pre=True, gate="channel", sig=False),
        # log-probabilities and loss of a few sampled tokens
        dict(name="policy_forward_few", op="policy", mode="forward", N=7, V=32768, dtype="bf16", tau=1.0, kl=0.0, ref=False, pad=0),
        # a policy step on a microbatch, large vocabulary, reference model beside it
        dict(name="policy_step_large", op="policy", mode="step", N=4096, V=131072, dtype="bf16", tau=1.0, kl=0.05, ref=True, pad=10),
        # loss and gradient in two calls (the losses are looked at between them), FP32, odd vocabulary, long prompts
        dict(name="policy_train_rows_f32", op="policy", mode="train", N=1023, V=100003, dtype="f32", tau=0.7, kl=0.1, ref=True, pad=40),
        # the gradients of a few low-rank adapters
        dict(name="clip_few", op="clip", sizes="65536 16384 128 65536 16384 128 196608 65536 1 777", src="f32", dst="bf16"),
        # FP32 accumulated gradients of the Qwen3-8B-shaped layer, clipped into the step's BF16 gradients
        dict(name="clip_layer_8b", op="clip", sizes="16777216 4194304 4194304 16777216 50331648 50331648 50331648 4096 4096 128 128",
             src="f32", dst="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "norm", "policy", "clip"])
    if op == "embed":
        V, dtype = _log_int(rng, 256, 131072), rng.choice(["bf16", "bf16", "f32"])
        H = rng.choice([_log_int(rng, 64, 4096), rng.choice([512, 1024, 2048, 4096])])
        T = _log_int(rng, 1, min(32768, 16384 * 4096 // H))
        grad = rng.choice([dtype, "f32"])
        if grad == "f32":
            V = min(V, 65536)
        return dict(op="embed", train=rng.random() < 0.6, T=T, V=V, H=H, dtype=dtype, grad=grad, pad=rng.choice([0, 0, 5, 30]))
    if op == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        H = rng.choice([_log_int(rng, 64, 8192), rng.choice([512, 1024, 2048, 4096, 5120, 8192])])
        T = _log_int(rng, 1, min(32768, 4096 * 4096 // H * (2 if dtype == "bf16" else 1)))
        post = rng.random() < 0.6
        return dict(op="norm", train=rng.random() < 0.6, T=T, H=H, dtype=dtype, post=post, pre=rng.random() < 0.85,
                    gate=rng.choice(["none", "none", "channel", "token"]), sig=rng.random() < 0.5)
    if op == "policy":
        V, dtype = _log_int(rng, 1000, 160000), rng.choice(["bf16", "bf16", "f32"])
        N = _log_int(rng, 1, min(8192, 4096 * 131072 // (V * (4 if dtype == "f32" else 1))))
        ref = rng.random() < 0.7
        return dict(op="policy", mode=rng.choice(["forward", "step", "train"]), N=N, V=V, dtype=dtype,
                    tau=rng.choice([1.0, 1.0, 0.7, 1.3]), kl=rng.choice([0.0, 0.02, 0.1]) if ref else 0.0, ref=ref, pad=rng.choice([0, 10, 40]))
    n = _log_int(rng, 1, 400)
    most = _log_int(rng, 100, (1 << 26) // n if n > 8 else 1 << 23)
    return dict(op="clip", sizes=" ".join(str(_log_int(rng, 1, most)) for _ in range(n)), src=rng.choice(["f32", "f32", "bf16"]), dst=rng.choice(["f32", "bf16"]))


# ---- inputs ------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 54321)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return {"embed": _prepare_embed, "norm": _prepare_norm, "policy": _prepare_policy, "clip": _prepare_clip}[case["op"]](case, g, rnd)


def _prepare_embed(c, g, rnd):
    T, V, H, dt = c["T"], c["V"], c["H"], _DTYPES[c["dtype"]]
    # token k is as frequent as 1 / k: the first ones make up much of a text
    ids = (float(V + 1) ** torch.rand(T, generator=g, device="cuda", dtype=F64)).long() - 1
    ids[T - T * c["pad"] // 100:] = -1
    s = dict(case=c, table=(0.02 * rnd(V, H)).to(dt), ids=ids.clamp(max=V - 1).to(torch.int32), scale=math.sqrt(H),
             out=torch.empty(T, H, dtype=dt, device="cuda"))
    if c["train"]:
        s.update(dy=(1e-3 * rnd(T, H)).to(dt), d_table=torch.empty(V, H, dtype=_DTYPES[c["grad"]], device="cuda"))
    return s


def _prepare_norm(c, g, rnd):
    T, H, dt = c["T"], c["H"], _DTYPES[c["dtype"]]
    new = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    s = dict(case=c, x=(2.0 * rnd(T, H)).to(dt), y=(0.7 * rnd(T, H)).to(dt), alpha=0.5, eps=1e-6,
             w_post=(1 + 0.1 * rnd(H)).to(dt) if c["post"] else None, w_pre=(1 + 0.1 * rnd(H)).to(dt) if c["pre"] else None,
             gate={"none": None, "channel": (0.5 + 0.3 * rnd(H)).to(dt), "token": rnd(T, H).to(dt)}[c["gate"]],
             x_out=new(T, H), h=new(T, H) if c["pre"] else None)
    if c["train"]:
        s.update(gx=rnd(T, H).to(dt), gh=rnd(T, H).to(dt) if c["pre"] else None, dx=new(T, H), dy=new(T, H),
                 dgate={"none": None, "channel": new(H, dtype=F32), "token": new(T, H)}[c["gate"]],
                 dw_post=new(H, dtype=F32) if c["post"] else None, dw_pre=new(H, dtype=F32) if c["pre"] else None)
    return s


_CLIP_LOW, _CLIP_HIGH = 0.2, 0.28


def _prompt(c):
    """Which rows have no label: the first `pad` hundredths of each of eight documents."""
    doc = max(1, c["N"] // 8)
    return torch.arange(c["N"]) % doc < doc * c["pad"] // 100


def _prepare_policy(c, g, rnd):
    N, V, dt, tau = c["N"], c["V"], _DTYPES[c["dtype"]], c["tau"]
    z = torch.empty(N, V, dtype=dt, device="cuda")
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    bias = 13.0 + 3.0 * rnd(N, 1)          # a sampled token is a likely one
    logp = torch.empty(N, dtype=F64, device="cuda")
    step = max(1, (1 << 27) // V)
    for lo in range(0, N, step):
        r = slice(lo, min(N, lo + step))
        z[r] = rnd(r.stop - lo, V) * 2.5
        z[r].scatter_(1, labels[r, None], bias[r].to(dt))
        zd = z[r].double() / tau
        logp[r] = zd.gather(1, labels[r, None])[:, 0] - torch.logsumexp(zd, 1)
    # the policy has moved a little since the tokens were sampled; no ratio lies on the edge of the clipped range to within FP32's digits
    moved = 0.25 * rnd(N).double()
    edge = torch.tensor([math.log1p(-_CLIP_LOW), math.log1p(_CLIP_HIGH)], device="cuda", dtype=F64)
    moved = torch.where(((moved[:, None] - edge).abs() < 1e-4).any(1), moved + 1e-3, moved)
    s = dict(case=c, z=z, labels=torch.where(_prompt(c).cuda(), -100, labels).to(torch.int32), old=(logp - moved).float(),
             ref=(logp + 0.3 * rnd(N)).float() if c["ref"] else None, adv=rnd(N), tau=tau, kl=c["kl"], loss=torch.empty(N, device="cuda"),
             logp=torch.empty(N, device="cuda"))
    if c["mode"] != "forward":
        s["dz"] = torch.empty_like(z)
        s["g"] = torch.rand(N, generator=g, device="cuda") / N
    return s


def _sizes(c):
    return [int(n) for n in c["sizes"].split()]


def _prepare_clip(c, g, rnd):
    sizes = _sizes(c)
    spread = 1e-3 * (1 + torch.rand(len(sizes), generator=g, device="cuda"))
    flat = torch.empty(sum(sizes), dtype=_DTYPES[c["dst"]], device="cuda")       # the step's gradient buffer
    return dict(case=c, grads=[(rnd(n) * spread[i]).to(_DTYPES[c["src"]]) for i, n in enumerate(sizes)],
                flat=flat, out=list(flat.split(sizes)), scale=0.25,
                most=0.1 * 1e-3 * math.sqrt(sum(sizes)), result=torch.empty(4, dtype=F64, device="cuda"))


# ---- one pass ----------------------------------------------------------------------------------

_ctx = None


def _context():
    global _ctx
    if _ctx is None:
        import paper_2609_34162_b200.slidedp as sd
        _ctx = sd.slidedp_create(torch.cuda.current_device(), 0)
    return _ctx


def run(state):
    op = state["case"]["op"]
    if own:
        return {"embed": _own_embed, "norm": _own_norm, "policy": _own_policy, "clip": _own_clip}[op](_context(), state)
    return {"embed": _plain_embed, "norm": _plain_norm, "policy": _plain_policy, "clip": _plain_clip}[op](state)


def _scratch(s, nbytes):
    """The program's workspace, made on the first pass."""
    if "ws" not in s:
        s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own_embed(ctx, s):
    ctx.slidedp_embedding(s["table"], s["ids"], s["out"], scale=s["scale"])
    if not s["case"]["train"]:
        return [s["out"]]
    ws = _scratch(s, ctx.slidedp_embedding_workspace(s["dy"], s["d_table"])) if "ws" not in s else s["ws"]
    ctx.slidedp_embedding_backward(s["ids"], s["dy"], s["d_table"], ws, scale=s["scale"])
    return [s["out"], s["d_table"]]


def _own_norm(ctx, s):
    how = dict(residual_scale=s["alpha"], eps=s["eps"], post_norm=s["case"]["post"], gate_sigmoid=s["case"]["sig"])
    ins = (s["x"], s["y"], s["w_post"], s["gate"], s["w_pre"])
    ctx.slidedp_block_norm(*ins, s["x_out"], s["h"], **how)
    out = [s["x_out"], s["h"]]
    if s["case"]["train"]:
        ws = _scratch(s, ctx.slidedp_block_norm_workspace(s["x"])) if "ws" not in s else s["ws"]
        ctx.slidedp_block_norm_backward(*ins, s["gx"], s["gh"], s["dx"], s["dy"], s["dgate"], s["dw_post"], s["dw_pre"], ws, **how)
        out += [s["dx"], s["dy"], s["dgate"], s["dw_post"], s["dw_pre"]]
    return [t for t in out if t is not None]


def _own_policy(ctx, s):
    how = dict(temperature=s["tau"], clip_low=_CLIP_LOW, clip_high=_CLIP_HIGH, kl_weight=s["kl"])
    ins = (s["z"], s["labels"], s["old"], s["ref"], s["adv"])
    if s["case"]["mode"] == "step":
        ctx.slidedp_policy_step(*ins, s["g"], s["loss"], s["logp"], s["dz"], **how)
        return [s["loss"], s["logp"], s["dz"]]
    ctx.slidedp_policy_loss(*ins, s["loss"], s["logp"], **how)
    if s["case"]["mode"] == "forward":
        return [s["loss"], s["logp"]]
    ctx.slidedp_policy_loss_backward(*ins, s["logp"], s["g"], s["dz"], **how)
    return [s["loss"], s["logp"], s["dz"]]


def _own_clip(ctx, s):
    ws = _scratch(s, ctx.slidedp_clip_grad_norm_workspace(s["grads"])) if "ws" not in s else s["ws"]
    ctx.slidedp_clip_grad_norm(s["grads"], s["out"], s["most"], s["result"], ws, scale=s["scale"])
    return [s["flat"], s["result"]]


# ---- the plain forms: 32 bits throughout, one rounding at the end --------------------------------

def _plain_embed(s):
    c, ids = s["case"], s["ids"].long()
    V, has = c["V"], (ids >= 0) & (ids < c["V"])
    out = torch.where(has[:, None], s["table"][ids.clamp(0, V - 1)].float() * s["scale"], 0.0).to(s["table"].dtype)
    if not c["train"]:
        return [out]
    total = torch.zeros(V + 1, c["H"], device=ids.device)
    total.index_add_(0, torch.where(has, ids, V), s["dy"].float())
    return [out, (total[:V] * s["scale"]).to(s["d_table"].dtype)]


def _plain_norm(s):
    c, dt, x, y = s["case"], s["x"].dtype, s["x"].float(), s["y"].float()
    one = torch.ones((), device=x.device)
    w_post, w_pre = (one if s[n] is None else s[n].float() for n in ("w_post", "w_pre"))
    gate = one if s["gate"] is None else s["gate"].float()
    turned = torch.sigmoid(gate) if c["sig"] and s["gate"] is not None else gate
    unit = lambda t: torch.rsqrt((t * t).mean(-1, keepdim=True) + s["eps"])  # noqa: E731
    r = unit(y) if c["post"] else one
    yh = y * r
    x2 = x + s["alpha"] * turned * (yh * w_post)
    r2 = unit(x2) if c["pre"] else one
    out = [x2.to(dt), (x2 * r2 * w_pre).to(dt) if c["pre"] else None]
    if c["train"]:
        d, dw_pre = s["gx"].float(), None
        if c["pre"]:
            gh, xh = s["gh"].float(), x2 * r2
            u = gh * w_pre
            d = d + r2 * (u - xh * (u * xh).mean(-1, keepdim=True))
            dw_pre = (gh * xh).sum(0)
        a = s["alpha"] * d
        v = a * turned * w_post
        dy = r * (v - yh * (v * yh).mean(-1, keepdim=True)) if c["post"] else v
        dw_post = (a * turned * yh).sum(0) if c["post"] else None
        dgate = None
        if s["gate"] is not None:
            dgate = a * yh * w_post * (turned * (1 - turned) if c["sig"] else one)
            dgate = dgate.sum(0) if c["gate"] == "channel" else dgate.to(dt)
        out += [d.to(dt), dy.to(dt), dgate, dw_post, dw_pre]
    return [t for t in out if t is not None]


def _plain_policy(s):
    c, z, tau = s["case"], s["z"].float(), s["tau"]
    V, lab = z.shape[1], s["labels"].long()
    has = (lab >= 0) & (lab < V)
    at = lab.clamp(0, V - 1)[:, None]
    top = z.amax(1, keepdim=True)
    e = ((z - top) / tau).exp_()
    total = e.sum(1, dtype=F64)
    # the ratio is compared with the edges of the clipped range: 64 bits per row
    logp = (z.gather(1, at) - top)[:, 0].double() / tau - total.log()
    ratio, adv = (logp - s["old"].double()).exp(), s["adv"].double()
    loss = -torch.minimum(ratio * adv, ratio.clamp(1 - _CLIP_LOW, 1 + _CLIP_HIGH) * adv)
    inside = torch.where(adv >= 0, ratio <= 1 + _CLIP_HIGH, ratio >= 1 - _CLIP_LOW)
    slope = torch.where(inside, -adv * ratio, 0.0)
    if s["ref"] is not None:
        k = s["ref"].double() - logp
        loss = loss + s["kl"] * (k.exp() - k - 1)
        slope = slope + s["kl"] * (1 - k.exp())
    out = [torch.where(has, loss, 0.0).float(), torch.where(has, logp, 0.0).float()]
    if c["mode"] != "forward":
        f = torch.where(has, slope * s["g"] / tau, 0.0)
        dz = e.mul_((-f / total).float()[:, None])
        dz.scatter_(1, at, (f * -torch.expm1(logp)).float()[:, None])
        out.append(dz.to(s["z"].dtype))
    return out


def _plain_clip(s):
    c = s["case"]
    flat = torch.cat(s["grads"])
    total = torch.linalg.vector_norm(flat, dtype=F64) ** 2 * s["scale"] ** 2
    norm = total.sqrt()
    coef = (s["most"] / (norm + 1e-6)).clamp(max=1.0)
    out = (flat.float() * (coef * s["scale"]).float()).to(_DTYPES[c["dst"]])
    return [out, torch.stack([total, norm, coef, 1.0 - norm.isfinite().double()])]


# ---- what a pass cannot do without ---------------------------------------------------------------

def _distinct(c):
    """Expected number of different tokens of a batch."""
    n, k, total = c["T"] - c["T"] * c["pad"] // 100, 0, 0.0
    whole = math.log(c["V"] + 1)
    while k < c["V"]:
        m = min(c["V"], max(k + 1, int(k * 1.05)))
        p = math.log((m + 1) / (k + 1)) / whole / (m - k)
        total += (m - k) * -math.expm1(n * math.log1p(-min(p, 1 - 1e-12)))
        k = m
    return total


def work(case):
    c = case
    if c["op"] == "embed":
        size, gsize, used = 4 if c["dtype"] == "f32" else 2, 4 if c["grad"] == "f32" else 2, _distinct(c)
        n, f = (used + c["T"]) * c["H"] * size + 4 * c["T"], c["T"] * c["H"]
        if c["train"]:
            n += c["T"] * (c["H"] * size + 4) + c["V"] * c["H"] * gsize
            f += (c["T"] + used) * c["H"]
        return {"bytes": int(n), "flops": f}
    if c["op"] == "norm":
        size, x = 4 if c["dtype"] == "f32" else 2, c["T"] * c["H"]
        token, pre = c["gate"] == "token", c["pre"]
        per = 3 + pre + token                                           # x, y, gate; x', h
        if c["train"]:
            per += 5 + pre + 2 * token                                  # x, y, gate, dx', dh; dx, dy, dgate
        return {"bytes": per * x * size + 16 * c["H"], "flops": (36 if c["train"] else 10) * x}
    if c["op"] == "policy":
        size, N, V = 4 if c["dtype"] == "f32" else 2, c["N"], c["V"]
        rows = N - int(_prompt(c).sum())
        reads, writes = {"forward": (1, 0), "step": (1, 1), "train": (2, 1)}[c["mode"]]
        return {"bytes": (reads * rows + writes * N) * V * size + 32 * N, "flops": (reads + writes) * 4 * rows * V}
    n, src, dst = sum(_sizes(c)), 4 if c["src"] == "f32" else 2, 4 if c["dst"] == "f32" else 2
    return {"bytes": n * (src + dst), "flops": 3 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "policy": _exact_policy, "clip": _exact_clip}[case["op"]](s)


def _exact_embed(s):
    """The table with a row of zeros at its end, which absent tokens select; the gradient by sorted tokens and differences of
    running sums over columns."""
    c, V = s["case"], s["case"]["V"]
    ids = torch.where(s["ids"] < 0, V, s["ids"].long())
    out = torch.cat([s["table"], s["table"].new_zeros(1, c["H"])]).index_select(0, ids).double().mul_(s["scale"])
    if not c["train"]:
        return [out]
    order = ids.argsort(stable=True)
    present, count = ids[order].unique_consecutive(return_counts=True)
    ends = count.cumsum(0)
    d = torch.zeros(V + 1, c["H"], dtype=F64, device="cuda")
    wide = max(1, (1 << 27) // c["T"])
    for lo in range(0, c["H"], wide):
        run = torch.nn.functional.pad(s["dy"][order, lo:lo + wide].double().cumsum(0), (0, 0, 1, 0))
        d[present, lo:lo + wide] = run[ends] - run[ends - count]
    return [out, d[:V] * s["scale"]]


def _exact_norm(s):
    """By automatic differentiation."""
    c = s["case"]
    leaf = {n: s[n].double().requires_grad_(c["train"]) for n in ("x", "y", "gate", "w_post", "w_pre") if s[n] is not None}

    def rms(t):
        return t / torch.sqrt(torch.linalg.vector_norm(t, dim=-1, keepdim=True) ** 2 / c["H"] + s["eps"])

    b = rms(leaf["y"]) * leaf["w_post"] if c["post"] else leaf["y"]
    if "gate" in leaf:
        b = b * (1 / (1 + torch.exp(-leaf["gate"])) if c["sig"] else leaf["gate"])
    x2 = leaf["x"] + s["alpha"] * b
    out, back = [x2], [s.get("gx")]
    if c["pre"]:
        out, back = out + [rms(x2) * leaf["w_pre"]], back + [s.get("gh")]
    if not c["train"]:
        return out
    grads = torch.autograd.grad(out, list(leaf.values()), [g.double() for g in back])
    return [t.detach() for t in out] + list(grads)


def _exact_policy(s):
    """A block of rows at a time, the slopes by automatic differentiation over the rows' log-probabilities."""
    c, tau = s["case"], s["tau"]
    N, V = c["N"], c["V"]
    loss, logp = torch.zeros(N, dtype=F64, device="cuda"), torch.zeros(N, dtype=F64, device="cuda")
    dz = torch.zeros(N, V, dtype=F64, device="cuda") if c["mode"] != "forward" else None
    step = max(1, (1 << 27) // V)
    for lo in range(0, N, step):
        rows = torch.arange(lo, min(N, lo + step), device="cuda")
        rows = rows[s["labels"][rows] >= 0]
        if not len(rows):
            continue
        lab = s["labels"][rows].long()
        z = torch.log_softmax(s["z"][rows].double() / tau, 1)
        lp = z[torch.arange(len(rows), device="cuda"), lab].requires_grad_()
        ratio, adv = torch.exp(lp - s["old"][rows].double()), s["adv"][rows].double()
        each = torch.maximum(-ratio * adv, -torch.clip(ratio, 1 - _CLIP_LOW, 1 + _CLIP_HIGH) * adv)
        if s["ref"] is not None:
            each = each + s["kl"] * (torch.expm1(s["ref"][rows].double() - lp) - (s["ref"][rows].double() - lp))
        loss[rows], logp[rows] = each.detach(), lp.detach()
        if dz is not None:
            f = torch.autograd.grad(each.sum(), lp)[0] * s["g"][rows].double() / tau
            d = torch.exp_(z).mul_(-f[:, None])
            d[torch.arange(len(rows), device="cuda"), lab] = -f * torch.expm1(lp.detach())
            dz[rows] = d
    return [loss, logp] + ([dz] if dz is not None else [])


def _exact_clip(s):
    total = sum((t.double() * s["scale"]).square().sum() for t in s["grads"])
    norm = torch.sqrt(total)
    coef = torch.clamp(s["most"] / (norm + 1e-6), max=1.0)
    return [torch.cat([t.double() * s["scale"] * coef for t in s["grads"]]), torch.stack([total, norm, coef, torch.zeros_like(coef)])]
