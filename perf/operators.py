"""Measured cases of the fine-tuning operators: query/key norms with the rotation, attention over
packed documents, and distillation from a teacher's top logits.

Each case runs in two forms on the same inputs: `own` false is elementary torch arithmetic in 32
bits, rounded once at the end; `own` true calls the library. ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
_DTYPES = {"bf16": BF16, "f32": F32}


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # one token at a time: what sampling from the model while it is being tuned asks for
        dict(name="qk_forward_one_token", op="qk", train=False, T=1, docs=1, Hq=32, Hk=8, D=128,
             rope=128, inter=False, dtype="bf16", fused=True),
        # a training microbatch through the Qwen3-8B-shaped layer (hidden 4096: 32 and 8 heads of 128)
        dict(name="qk_train_8b", op="qk", train=True, T=8192, docs=9, Hq=32, Hk=8, D=128,
             rope=128, inter=False, dtype="bf16", fused=True),
        # a long forward pass (evaluation) through the Qwen3-14B-shaped layer (hidden 5120: 40 heads)
        dict(name="qk_forward_14b_long", op="qk", train=False, T=16384, docs=1, Hq=40, Hk=8, D=128,
             rope=128, inter=False, dtype="bf16", fused=True),
        # small model tuned in FP32: odd token count, part of each head rotated, interleaved pairs
        dict(name="qk_train_partial_f32", op="qk", train=True, T=1537, docs=3, Hq=12, Hk=4, D=80,
             rope=48, inter=True, dtype="f32", fused=False),
        # a single short sample
        dict(name="attn_forward_short", op="attn", train=False, T=77, docs=1, pad=0, Hq=8, Hk=2, D=64,
             causal=True, prefix=False, cap=0.0, bias=False),
        # evaluation over a packed batch of documents, Qwen3-8B-shaped heads
        dict(name="attn_forward_packed_8b", op="attn", train=False, T=8192, docs=11, pad=100, Hq=32, Hk=8,
             D=128, causal=True, prefix=False, cap=0.0, bias=False),
        # a training microbatch that is one long document: the largest attention
        dict(name="attn_train_long_8b", op="attn", train=True, T=8192, docs=1, pad=0, Hq=32, Hk=8, D=128,
             causal=True, prefix=False, cap=0.0, bias=False),
        # packed prompt/answer pairs (each prompt sees itself whole), capped scores, distance bias,
        # an odd token count and a padded end
        dict(name="attn_train_prefix_cap_bias", op="attn", train=True, T=4099, docs=7, pad=45, Hq=16, Hk=4,
             D=96, causal=True, prefix=True, cap=30.0, bias=True),
        # the loss on a handful of held-out tokens
        dict(name="distill_forward_few", op="distill", mode="forward", N=7, V=32768, K=8, tau=1.0,
             wt=1.0, wl=0.0, dtype="bf16", pad=0),
        # loss and gradient of a training microbatch over a large vocabulary
        dict(name="distill_step_large", op="distill", mode="step", N=4096, V=131072, K=64, tau=2.0,
             wt=1.0, wl=0.0, dtype="bf16", pad=0),
        # FP32 logits, a vocabulary no vector width divides, hard labels mixed in, padded entries
        dict(name="distill_step_mixed_f32", op="distill", mode="step", N=1023, V=100003, K=20, tau=1.5,
             wt=0.7, wl=0.3, dtype="f32", pad=3),
        # forward and, later, backward with a gradient per row (a loss that is weighted afterwards)
        dict(name="distill_train_rows", op="distill", mode="train", N=2048, V=50257, K=32, tau=1.0,
             wt=0.5, wl=0.5, dtype="bf16", pad=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qk", "attn", "distill"])
    if op == "qk":
        Hk = rng.choice([1, 2, 4, 8])
        Hq = min(64, Hk * rng.choice([1, 3, 4, 5, 8]))
        D = rng.choice([64, 80, 96, 128, 256])
        rope = rng.choice([D, D, D, D // 2])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = 40 * 16384 * 128 // ((Hq + Hk) * D * (2 if dtype == "f32" else 1))
        T = _log_int(rng, 1, min(16384, most))
        return dict(op="qk", train=rng.random() < 0.5, T=T, docs=rng.randint(1, min(T, 12)), Hq=Hq, Hk=Hk,
                    D=D, rope=rope, inter=rng.random() < 0.3, dtype=dtype, fused=rng.random() < 0.7)
    if op == "attn":
        Hk = rng.choice([1, 2, 4, 8])
        Hq = min(32, Hk * rng.choice([1, 2, 4, 5, 8]))
        D = rng.choice([64, 80, 96, 128])
        T = _log_int(rng, 1, 7000)
        return dict(op="attn", train=rng.random() < 0.5, T=T, docs=rng.randint(1, min(T, 12)),
                    pad=rng.choice([0, 0, T // 10]), Hq=Hq, Hk=Hk, D=D, causal=rng.random() < 0.8,
                    prefix=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.3)
    V = _log_int(rng, 1000, 160000)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    N = _log_int(rng, 1, max(2, 4096 * 131072 // (V * (2 if dtype == "f32" else 1))) if V > 65536 else 4096)
    wt = rng.choice([1.0, 1.0, 0.5, 0.0])
    return dict(op="distill", mode=rng.choice(["forward", "step", "train"]), N=N, V=V, K=rng.choice([1, 8, 20, 64, 100]),
                tau=rng.choice([1.0, 2.0, 3.5]), wt=wt, wl=1.0 - wt, dtype=dtype, pad=rng.choice([0, 0, 1]))


# ---- inputs ------------------------------------------------------------------------------------

def _doc_offsets(case):
    """Document offsets that the case alone decides (so that its work is known): ascending, the
    tokens after the last one are padding."""
    total, docs = case["T"] - case.get("pad", 0), case["docs"]
    r = random.Random(1000003 * case["T"] + 97 * docs)
    docs = min(docs, total)
    return [0] + sorted(r.sample(range(1, total), docs - 1)) + [total] if docs > 1 else [0, total]


def _prefixes(case):
    """Prompt length of each document: about a third of it, sometimes none."""
    off, r = _doc_offsets(case), random.Random(case["T"])
    return [0 if r.random() < 0.2 else (b - a) * r.randint(1, 60) // 100 for a, b in zip(off, off[1:])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 12345)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return {"qk": _prepare_qk, "attn": _prepare_attn, "distill": _prepare_distill}[case["op"]](case, g, rnd)


def _prepare_qk(c, g, rnd):
    T, Hq, Hk, D, dt = c["T"], c["Hq"], c["Hk"], c["D"], _DTYPES[c["dtype"]]
    if c["fused"]:        # the views of one projection's output, values beside them
        qkv = (rnd(T, Hq + 2 * Hk, D) * 1.5).to(dt)
        q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    else:
        q, k = (rnd(T, Hq, D) * 1.5).to(dt), (rnd(T, Hk, D) * 1.5).to(dt)
    off = torch.tensor(_doc_offsets(c), device="cuda")
    t = torch.arange(T, device="cuda")
    pos = (t - off[torch.searchsorted(off, t, right=True) - 1]).to(torch.int32)   # restarts per document
    half = c["rope"] // 2
    inv = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    ang = torch.arange(T, device="cuda", dtype=torch.float64)[:, None] * inv
    s = dict(case=c, q=q, k=k, wq=(1 + 0.1 * rnd(D)).to(dt), wk=(1 + 0.1 * rnd(D)).to(dt), pos=pos,
             cos_sin=torch.cat([ang.cos(), ang.sin()], 1).to(F32), eps=1e-6,
             yq=torch.empty(T, Hq, D, dtype=dt, device="cuda"), yk=torch.empty(T, Hk, D, dtype=dt, device="cuda"))
    if c["train"]:
        s.update(gq=rnd(T, Hq, D).to(dt), gk=rnd(T, Hk, D).to(dt),
                 dq=torch.empty(T, Hq, D, dtype=dt, device="cuda"), dk=torch.empty(T, Hk, D, dtype=dt, device="cuda"),
                 dwq=torch.empty(D, device="cuda"), dwk=torch.empty(D, device="cuda"))
    return s


def _prepare_attn(c, g, rnd):
    T, Hq, Hk, D = c["T"], c["Hq"], c["Hk"], c["D"]
    q, k = rnd(T, Hq, D).to(BF16), rnd(T, Hk, D).to(BF16)
    v = rnd(T, Hq + 2 * Hk, D).to(BF16)[:, Hq + Hk:]        # the values' view of the projection's output
    s = dict(case=c, q=q, k=k, v=v, scale=D ** -0.5, cap=c["cap"], causal=c["causal"],
             cu=torch.tensor(_doc_offsets(c), dtype=torch.int32, device="cuda"),
             prefix=torch.tensor(_prefixes(c), dtype=torch.int32, device="cuda") if c["prefix"] else None,
             slopes=2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if c["bias"] else None,
             out=torch.empty(T, Hq, D, dtype=BF16, device="cuda"), lse=torch.empty(Hq, T, device="cuda"))
    if c["train"]:
        s.update(do=rnd(T, Hq, D).to(BF16), dq=torch.empty(T, Hq, D, dtype=BF16, device="cuda"),
                 dk=torch.empty(T, Hk, D, dtype=BF16, device="cuda"), dv=torch.empty(T, Hk, D, dtype=BF16, device="cuda"))
    return s


def _prepare_distill(c, g, rnd):
    N, V, K, dt = c["N"], c["V"], c["K"], _DTYPES[c["dtype"]]
    z = torch.empty(N, V, dtype=dt, device="cuda")
    step = max(1, (1 << 27) // V)
    for lo in range(0, N, step):
        z[lo:lo + step] = rnd(min(step, N - lo), V) * 2.5
    # K different entries of each row, their logits falling from the first; the student half agrees
    ids = (torch.randint(0, V, (N, 1), generator=g, device="cuda")
           + torch.arange(K, device="cuda") * max(1, V // (2 * K) | 1)) % V
    t = 8.0 - 0.25 * torch.arange(K, device="cuda") + 0.2 * rnd(N, K)
    z.scatter_(1, ids, (0.7 * t + rnd(N, K)).to(dt))
    if c["pad"]:          # fewer entries than the table is wide; one row in 16 has none
        ids[:, K - min(c["pad"], K - 1):] = -1 if K > 1 else ids[:, :1]
        ids[::16] = -1
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    labels[torch.rand(N, generator=g, device="cuda") < 0.1] = -100            # prompt tokens
    s = dict(case=c, z=z, ids=ids.to(torch.int32), t=t, labels=labels.to(torch.int32), tau=c["tau"], wt=c["wt"],
             wl=c["wl"], loss=torch.empty(N, device="cuda"), lse=torch.empty(2, N, device="cuda"))
    if c["mode"] != "forward":
        s["dz"] = torch.empty_like(z)
        s["g"] = torch.rand(N, generator=g, device="cuda") / N
    return s


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
        return {"qk": _own_qk, "attn": _own_attn, "distill": _own_distill}[op](_context(), state)
    return {"qk": _plain_qk, "attn": _plain_attn, "distill": _plain_distill}[op](state)


def _own_qk(ctx, s):
    c = s["case"]
    rope = dict(eps=s["eps"], interleaved=c["inter"])
    ctx.slidedp_qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos_sin"], s["pos"], s["yq"], s["yk"], **rope)
    out = [s["yq"], s["yk"]]
    if c["train"]:
        if "ws" not in s:
            s["ws"] = torch.empty(ctx.slidedp_qk_norm_rope_workspace(s["q"], s["k"]), dtype=torch.uint8, device="cuda")
        ctx.slidedp_qk_norm_rope_backward(s["q"], s["k"], s["wq"], s["wk"], s["cos_sin"], s["pos"], s["gq"], s["gk"],
                                          s["dq"], s["dk"], s["dwq"], s["dwk"], s["ws"], **rope)
        out += [s["dq"], s["dk"], s["dwq"], s["dwk"]]
    return out


def _own_attn(ctx, s):
    mask = dict(cu_docs=s["cu"], prefix=s["prefix"], slopes=s["slopes"], causal=s["causal"], scale=s["scale"],
                softcap=s["cap"])
    ctx.slidedp_attention(s["q"], s["k"], s["v"], s["out"], s["lse"], **mask)
    out = [s["out"], s["lse"]]
    if s["case"]["train"]:
        if "ws" not in s:
            s["ws"] = torch.empty(ctx.slidedp_attention_workspace(s["q"], s["k"]), dtype=torch.uint8, device="cuda")
        ctx.slidedp_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"],
                                       s["ws"], **mask)
        out += [s["dq"], s["dk"], s["dv"]]
    return out


def _own_distill(ctx, s):
    mix = dict(temperature=s["tau"], w_teacher=s["wt"], w_label=s["wl"])
    ins = (s["z"], s["ids"], s["t"], s["labels"])
    if s["case"]["mode"] == "step":
        ctx.slidedp_distill_step(*ins, s["g"], s["loss"], s["lse"], s["dz"], **mix)
        return [s["loss"], s["lse"], s["dz"]]
    ctx.slidedp_distill_loss(*ins, s["loss"], s["lse"], **mix)
    if s["case"]["mode"] == "forward":
        return [s["loss"], s["lse"]]
    ctx.slidedp_distill_loss_backward(*ins, s["lse"], s["g"], s["dz"], **mix)
    return [s["loss"], s["lse"], s["dz"]]


# ---- the plain forms: 32 bits throughout, one rounding at the end --------------------------------

def _split(x, rope, inter):
    """First and second members of the rotated pairs, and the rest of the head."""
    r, rest = x[..., :rope], x[..., rope:]
    return (r[..., 0::2], r[..., 1::2], rest) if inter else (r[..., :rope // 2], r[..., rope // 2:], rest)


def _join(a, b, rest, inter):
    r = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def _rotate(x, cos, sin, inter):
    a, b, rest = _split(x, 2 * cos.shape[-1], inter)
    return _join(a * cos - b * sin, b * cos + a * sin, rest, inter)


def _plain_qk(s):
    c = s["case"]
    row = s["cos_sin"][s["pos"].long()][:, None, :]
    cos, sin = row.chunk(2, -1)

    def forward(x, w):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
        return _rotate(x * r * w.float(), cos, sin, c["inter"])

    def backward(x, w, dy):
        x, w = x.float(), w.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
        dz, xh = _rotate(dy.float(), cos, -sin, c["inter"]), x * r
        u = dz * w
        return r * (u - xh * (u * xh).mean(-1, keepdim=True)), (dz * xh).sum((0, 1))

    dt = s["q"].dtype
    out = [forward(s["q"], s["wq"]).to(dt), forward(s["k"], s["wk"]).to(dt)]
    if c["train"]:
        dq, dwq = backward(s["q"], s["wq"], s["gq"])
        dk, dwk = backward(s["k"], s["wk"], s["gk"])
        out += [dq.to(dt), dk.to(dt), dwq, dwk]
    return out


def _visible(s, T):
    """[T, T] truth values: which keys (columns) each query (row) sees."""
    cu = s["cu"].long()
    t = torch.arange(T, device="cuda")
    doc = torch.searchsorted(cu, t, right=True) - 1
    ok = (doc[:, None] == doc[None, :]) & (t < cu[-1])[None, :]
    if s["causal"]:
        see = t[None, :] <= t[:, None]
        if s["prefix"] is not None:
            d = doc.clamp(max=len(cu) - 2)
            see = see | (t - cu[d] < s["prefix"].long()[d])[None, :]
        ok = ok & see
    return ok, t


def _plain_attn(s):
    q, k, v = (s[n].float().transpose(0, 1) for n in "qkv")          # [H, T, D]
    Hq, T, D = q.shape
    Hk = k.shape[0]
    ok, t = _visible(s, T)
    q4 = q.view(Hk, Hq // Hk, T, D)
    k4, v4 = k[:, None], v[:, None]
    x = (q4 @ k4.transpose(-1, -2)).mul_(s["scale"])
    th = torch.tanh(x / s["cap"]) if s["cap"] else None
    if th is not None:
        x = s["cap"] * th
    if s["slopes"] is not None:
        x = x - s["slopes"].view(Hk, Hq // Hk, 1, 1) * (t[:, None] - t[None, :]).abs()
    x = x.masked_fill_(~ok, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0))
    o = p @ v4
    lse = (m + total.log()).view(Hq, T)
    heads = lambda y, H: y.reshape(H, T, D).transpose(0, 1).contiguous().to(BF16)  # noqa: E731
    out = [heads(o, Hq), lse]
    if s["case"]["train"]:
        do = s["do"].float().transpose(0, 1).view(Hk, Hq // Hk, T, D)
        dv = (p.transpose(-1, -2) @ do).sum(1)
        dp = do @ v4.transpose(-1, -2)
        ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
        if th is not None:
            ds = ds * (1 - th * th)
        ds = ds * s["scale"]
        out += [heads(ds @ k4, Hq), heads((ds.transpose(-1, -2) @ q4).sum(1), Hk), heads(dv, Hk)]
    return out


def _plain_distill(s):
    c, z = s["case"], s["z"].float()
    N, V = z.shape
    tau, wt, wl = s["tau"], s["wt"], s["wl"]
    ids, lab = s["ids"].long(), s["labels"].long()
    has, hard = (ids >= 0) & (ids < V), (lab >= 0) & (lab < V)
    loss = torch.zeros(N, device=z.device)
    zero = torch.zeros(N, device=z.device)
    at = ids.clamp(0, V - 1)
    t = (s["t"].float() / tau).masked_fill(~has, -math.inf)
    some = has.any(1)
    m = torch.where(some, t.amax(1), 0.0)
    e = (t - m[:, None]).exp()
    qs = e.sum(1)
    q = e / torch.where(some, qs, 1.0)[:, None]
    logq = torch.where(has, t - m[:, None] - torch.where(some, qs, 1.0).log()[:, None], 0.0)
    zm = z.amax(1)
    lse_tau = zm / tau + ((z - zm[:, None]) / tau).exp().sum(1).log()
    lse_one = zm + (z - zm[:, None]).exp().sum(1).log() if wl else zero
    logp = z.gather(1, at) / tau - lse_tau[:, None]
    loss = loss + wt * tau * tau * (q * (logq - logp)).sum(1)
    if wl:
        nll = lse_one - z.gather(1, lab.clamp(0, V - 1)[:, None])[:, 0]
        loss = loss + wl * torch.where(hard, nll, 0.0)
    out = [loss, torch.stack([lse_tau, lse_one])]
    if c["mode"] != "forward":
        a = s["g"] * wt * tau * some
        dz = (z / tau - lse_tau[:, None]).exp_() * a[:, None]
        dz.scatter_add_(1, at, -a[:, None] * q)
        if wl:
            b = s["g"] * wl * hard
            dz += (z - lse_one[:, None]).exp_() * b[:, None]
            dz.scatter_add_(1, lab.clamp(0, V - 1)[:, None], -b[:, None])
        out.append(dz.to(s["z"].dtype))
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------

def _pairs(c):
    off, total = _doc_offsets(c), 0
    pre = _prefixes(c) if c["prefix"] else [0] * (len(off) - 1)
    for a, b, p in zip(off, off[1:], pre):
        n = b - a
        total += n * (n + 1) // 2 + p * (p - 1) // 2 if c["causal"] else n * n
    return total


def work(case):
    c = case
    if c["op"] == "qk":
        size = 4 if c["dtype"] == "f32" else 2
        x = c["T"] * (c["Hq"] + c["Hk"]) * c["D"]
        table = c["T"] * (4 * c["rope"] + 4)
        per = (2 + 3) if c["train"] else 2          # x, y; then x, dy, dx
        n = (2 if c["train"] else 1)
        return {"bytes": per * x * size + n * (table + 2 * c["D"] * size) + (8 * c["D"] if c["train"] else 0),
                "flops": (26 if c["train"] else 9) * x}
    if c["op"] == "attn":
        q, k = c["T"] * c["Hq"] * c["D"] * 2, c["T"] * c["Hk"] * c["D"] * 2
        lse = 4 * c["T"] * c["Hq"]
        n = 2 * q + 2 * k + lse
        if c["train"]:                              # q, k, v, o, do, lse again; dq, dk, dv
            n += 3 * q + 2 * k + lse + q + 2 * k
        return {"bytes": n, "flops": (14 if c["train"] else 4) * _pairs(c) * c["Hq"] * c["D"]}
    size = 4 if c["dtype"] == "f32" else 2
    z = c["N"] * c["V"] * size
    reads = {"forward": 1, "step": 1, "train": 2}[c["mode"]]
    writes = 0 if c["mode"] == "forward" else 1
    exps = 2 if c["wl"] else 1
    return {"bytes": (reads + writes) * z + c["N"] * (8 * c["K"] + 24), "flops": (reads + writes) * 4 * exps * c["N"] * c["V"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"qk": _exact_qk, "attn": _exact_attn, "distill": _exact_distill}[case["op"]](s)


def _exact_qk(s):
    """With the rotation as multiplication by exp(i angle) and the gradient by automatic differentiation."""
    c = s["case"]
    half = c["rope"] // 2
    cs = s["cos_sin"].double()[s["pos"].long()]
    turn = torch.complex(cs[:, :half].contiguous(), cs[:, half:].contiguous())[:, None]
    pair = torch.arange(c["rope"], device="cuda").view(half, 2) if c["inter"] else torch.arange(c["rope"], device="cuda").view(2, half).T

    def forward(x, w):
        n = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["D"] + s["eps"]) * w
        z = torch.complex(n[..., pair[:, 0]], n[..., pair[:, 1]]) * turn
        return n.index_copy(-1, pair[:, 0], z.real).index_copy(-1, pair[:, 1], z.imag)

    out, grads = [], []
    for n in ("q", "k"):
        x = s[n].double().requires_grad_(c["train"])
        w = s["w" + n].double().requires_grad_(c["train"])
        y = forward(x, w)
        out.append(y.detach())
        if c["train"]:
            grads.append(torch.autograd.grad(y, (x, w), s["g" + n].double()))
    return out + [g[0] for g in grads] + [g[1] for g in grads]


def _exact_attn(s):
    """Head by head, document by document."""
    c, T, D = s["case"], s["case"]["T"], s["case"]["D"]
    G = c["Hq"] // c["Hk"]
    z = lambda H: torch.zeros(T, H, D, dtype=torch.float64, device="cuda")  # noqa: E731
    o, dq, dk, dv = z(c["Hq"]), z(c["Hq"]), z(c["Hk"]), z(c["Hk"])
    lse = torch.full((c["Hq"], T), -math.inf, dtype=torch.float64, device="cuda")
    off = s["cu"].tolist()
    pre = s["prefix"].tolist() if s["prefix"] is not None else [0] * len(off)
    for (a, b), p in zip(zip(off, off[1:]), pre):
        i = torch.arange(b - a, device="cuda")
        hide = (i[None, :] > i[:, None]) & (i[None, :] >= p) if c["causal"] else None
        for h in range(c["Hq"]):
            q, k, v = s["q"][a:b, h].double(), s["k"][a:b, h // G].double(), s["v"][a:b, h // G].double()
            x = q @ k.T * s["scale"]
            slope = 1.0
            if s["cap"]:
                x = s["cap"] * torch.tanh(x / s["cap"])
                slope = 1.0 - (x / s["cap"]) ** 2
            if s["slopes"] is not None:
                x = x - float(s["slopes"][h]) * (i[:, None] - i[None, :]).abs()
            if hide is not None:
                x.masked_fill_(hide, -math.inf)
            L = torch.logsumexp(x, 1)
            P = torch.exp(x - L[:, None])
            lse[h, a:b], o[a:b, h] = L, P @ v
            if c["train"]:
                do = s["do"][a:b, h].double()
                dP = do @ v.T
                dS = P * (dP - (P * dP).sum(1, keepdim=True)) * slope * s["scale"]
                dq[a:b, h] = dS @ k
                dk[a:b, h // G] += dS.T @ q
                dv[a:b, h // G] += P.T @ do
    return [o, lse] + ([dq, dk, dv] if c["train"] else [])


def _exact_distill(s):
    """A block of rows at a time, the teacher's distribution written out over the vocabulary."""
    c = s["case"]
    N, V, tau = c["N"], c["V"], s["tau"]
    loss = torch.empty(N, dtype=torch.float64, device="cuda")
    lse = torch.zeros(2, N, dtype=torch.float64, device="cuda")
    dz = torch.empty(N, V, dtype=torch.float64, device="cuda") if c["mode"] != "forward" else None
    step = max(1, (1 << 28) // V)
    for lo in range(0, N, step):
        r = slice(lo, min(N, lo + step))
        z = s["z"][r].double()
        n = z.shape[0]
        logp = torch.log_softmax(z / tau, 1)
        lse[0, r] = torch.logsumexp(z / tau, 1)
        ids = s["ids"][r].long()
        has = ids >= 0
        t = torch.where(has, s["t"][r].double() / tau, -math.inf)
        q = torch.where(has, torch.exp(t - torch.where(has.any(1, keepdim=True), torch.logsumexp(t, 1, keepdim=True), 0.0)), 0.0)
        whole = torch.zeros(n, V + 1, dtype=torch.float64, device="cuda")
        whole.scatter_add_(1, torch.where(has, ids, V), q)
        whole = whole[:, :V]
        entropy = torch.special.entr(q).sum(1)          # ids differ within a row
        loss[r] = c["wt"] * tau ** 2 * (-entropy - (whole * logp).sum(1))
        if dz is not None:
            dz[r] = c["wt"] * tau * (torch.exp(logp) * whole.sum(1, keepdim=True) - whole)
        if c["wl"]:
            lse[1, r] = torch.logsumexp(z, 1)
            lab = s["labels"][r].long()
            hard = (lab >= 0).double()
            one = torch.zeros_like(z).scatter_(1, lab.clamp(min=0)[:, None], 1.0)
            logs = z - lse[1, r][:, None]
            loss[r] -= c["wl"] * hard * (one * logs).sum(1)
            if dz is not None:
                dz[r] += c["wl"] * hard[:, None] * (torch.exp(logs) - one)
        if dz is not None:
            dz[r] *= s["g"][r].double()[:, None]
    return [loss, lse] + ([dz] if dz is not None else [])
