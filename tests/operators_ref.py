"""The fine-tuning operators written out in 64 bits, row by row where that is plainest, for the parity
tests: no code, constant or layout of the library is used here. Every function works on CPU or GPU
tensors and returns float64."""
from __future__ import annotations

import math

import torch


# ---- norm and rotation of one [T, H, D] tensor ---------------------------------------------------

def qk_forward(x, w, cos_sin, pos, eps, interleaved):
    x = x.double()
    T, H, D = x.shape
    w = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
    n = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + eps) * w
    if cos_sin is None:
        return n
    rope = cos_sin.shape[1]
    half = rope // 2
    y = n.clone()
    for p in range(half):
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
        c, s = (cos_sin.double()[pos.long(), i][:, None] for i in (p, half + p))
        y[..., a] = n[..., a] * c - n[..., b] * s
        y[..., b] = n[..., b] * c + n[..., a] * s
    return y


def qk_backward(x, w, cos_sin, pos, eps, interleaved, dy):
    """(dx, dw) by the formula: dz = R^T dy, u = w dz, dx = r (u - xh mean(u xh)), dw = sum dz xh."""
    x, dz = x.double(), dy.double().clone()
    D = x.shape[-1]
    w = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
    if cos_sin is not None:
        half = cos_sin.shape[1] // 2
        for p in range(half):
            a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
            c, s = (cos_sin.double()[pos.long(), i][:, None] for i in (p, half + p))
            ga, gb = dy.double()[..., a], dy.double()[..., b]
            dz[..., a] = ga * c + gb * s
            dz[..., b] = gb * c - ga * s
    r = 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / D + eps)
    xh, u = x * r, w * dz
    return r * (u - xh * (u * xh).mean(-1, keepdim=True)), (dz * xh).sum((0, 1))


# ---- attention over packed documents --------------------------------------------------------------

def visible(T, cu, prefix, causal, device="cpu"):
    """[T, T] truth values, query by key, straight from the definition."""
    ok = torch.zeros(T, T, dtype=torch.bool)
    cu = [0, T] if cu is None else [int(c) for c in cu]
    for d, (a, b) in enumerate(zip(cu, cu[1:])):
        for i in range(a, b):
            if causal:
                ok[i, a:i + 1] = True
                if prefix is not None and int(prefix[d]) > 0:
                    ok[i, a:min(b, a + int(prefix[d]))] = True
            else:
                ok[i, a:b] = True
    return ok.to(device)


def attention(q, k, v, scale, ok, softcap=0.0, slopes=None, do=None):
    """out, lse and, with `do`, (dq, dk, dv) and elementwise bounds of what rounding the probabilities
    and the score gradients to BF16, and the saved out, can move each of them by."""
    T, Hq, D = q.shape
    Hk = k.shape[1]
    G = Hq // Hk
    dev = q.device
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros_like(q), torch.full((Hq, T), -math.inf, dtype=torch.float64, device=dev)
    res = {"out": out, "lse": lse, "out_bound": torch.zeros_like(q)}
    if do is not None:
        do = do.double()
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            res[n], res[n + "_bound"] = torch.zeros_like(x), torch.zeros_like(x)
    dist = (torch.arange(T, device=dev)[:, None] - torch.arange(T, device=dev)[None, :]).abs().double()
    u = 2.0 ** -8       # BF16 has 8 significant bits: rounding moves a value of [1, 2) by up to 2^-8
    for h in range(Hq):
        kk, vv = k[:, h // G], v[:, h // G]
        s = q[:, h] @ kk.T * scale
        grad = torch.ones_like(s)
        if softcap:
            th = torch.tanh(s / softcap)
            s, grad = softcap * th, 1 - th * th
        if slopes is not None:
            s = s - float(slopes[h]) * dist
        s = torch.where(ok, s, -math.inf)
        some = ok.any(1)
        L = torch.where(some, torch.logsumexp(s, 1), 0.0)
        p = torch.where(ok, torch.exp(s - L[:, None]), 0.0)
        lse[h] = torch.where(some, L, -math.inf)
        out[:, h] = p @ vv
        res["out_bound"][:, h] = u * (p @ vv.abs())
        if do is not None:
            g = do[:, h]
            dp = g @ vv.T
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta) * grad * scale
            res["dq"][:, h] = ds @ kk
            res["dk"][:, h // G] += ds.T @ q[:, h]
            res["dv"][:, h // G] += p.T @ g
            # |error of delta| <= u sum_d |do| |out| (out is rounded), and out's own error
            slack = ((g.abs() * (out[:, h].abs() * u + res["out_bound"][:, h])).sum(1, keepdim=True))
            es = u * ds.abs() + p * slack * grad * abs(scale)
            res["dq_bound"][:, h] = es @ kk.abs()
            res["dk_bound"][:, h // G] += es.T @ q[:, h].abs()
            res["dv_bound"][:, h // G] += u * (p.T @ g.abs())
    return res


# ---- distillation ----------------------------------------------------------------------------------

def distill(z, ids, t, labels, tau, wt, wl, row_grad=None):
    """loss [N], lse [2, N] and dz [N, V], one row at a time."""
    z, t = z.double(), t.double()
    N, V = z.shape
    loss, lse = torch.zeros(N, dtype=torch.float64), torch.zeros(2, N, dtype=torch.float64)
    dz = torch.zeros(N, V, dtype=torch.float64)
    z, t = z.cpu(), t.cpu()
    for r in range(N):
        g = 1.0 if row_grad is None else float(row_grad[r])
        have = [(int(i), float(x)) for i, x in zip(ids[r].tolist(), t[r].tolist()) if 0 <= i < V]
        lse[0, r] = torch.logsumexp(z[r] / tau, 0)
        top = max((x for _, x in have), default=-math.inf)
        if top > -math.inf:
            e = [math.exp((x - top) / tau) for _, x in have]
            q = [x / sum(e) for x in e]
            logp = z[r] / tau - lse[0, r]
            p = torch.exp(logp)
            for (i, _), qi in zip(have, q):
                if qi > 0.0:
                    loss[r] += wt * tau * tau * qi * (math.log(qi) - float(logp[i]))
                    dz[r, i] -= g * wt * tau * qi
            dz[r] += g * wt * tau * p
        if wl != 0.0 and labels is not None:
            lse[1, r] = torch.logsumexp(z[r], 0)
            y = int(labels[r])
            if 0 <= y < V:
                loss[r] += wl * float(lse[1, r] - z[r, y])
                dz[r] += g * wl * torch.exp(z[r] - lse[1, r])
                dz[r, y] -= g * wl
    return loss, lse, dz
