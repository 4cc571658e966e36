"""Token embedding, the norms around a block, the clipped policy loss and clipping over many tensors, written out in 64 bits for the
parity tests: no code, constant or layout of the library is used here. Beside each result stands the sum of the absolute terms
that it is made of, which rounding errors are relative to. Every function works on CPU or GPU tensors and returns float64."""
from __future__ import annotations

import math

import torch

F64 = torch.float64


def embedding(table, ids, scale):
    out = torch.zeros(len(ids), table.shape[1], dtype=F64, device=table.device)
    for t, i in enumerate(ids.tolist()):
        if 0 <= i < table.shape[0]:
            out[t] = scale * table[i].double()
    return out


def embedding_backward(ids, d_out, vocab, scale, before=None):
    """d_table, sum of absolute terms, terms per row."""
    d = torch.zeros(vocab, d_out.shape[1], dtype=F64, device=d_out.device)
    size, count = torch.zeros_like(d), torch.zeros(vocab, 1, dtype=F64, device=d_out.device)
    ok = (ids >= 0) & (ids < vocab)
    i = ids[ok].long()
    d.index_add_(0, i, scale * d_out[ok].double())
    size.index_add_(0, i, abs(scale) * d_out[ok].double().abs())
    count.index_add_(0, i, torch.ones(len(i), 1, dtype=F64, device=d_out.device))
    if before is not None:
        d, size = d + before.double(), size + before.double().abs()
    return d, size, count


def block_norm(x, y, w_post, gate, w_pre, alpha, eps, post, sigmoid, dx_out=None, dh=None, pre=True, backward=False):
    """A dict of the results, and under name + "_size" the absolute terms of each."""
    x = x.double()
    H = x.shape[1]
    one = torch.ones((), dtype=F64, device=x.device)
    dbl = lambda t: one if t is None else t.double()  # noqa: E731
    w_post, w_pre = dbl(w_post if post else None), dbl(w_pre)
    res = {}
    if y is not None:
        y = y.double()
        r = 1 / torch.sqrt((y * y).sum(1, keepdim=True) / H + eps) if post else one
        n = y * r * w_post
        g = dbl(gate)
        slope = torch.ones_like(g)
        if gate is not None and sigmoid:
            g = 1 / (1 + torch.exp(-g))
            slope = g * (1 - g)
        x2 = x + alpha * g * n
        res["x_out"], res["x_out_size"] = x2, x.abs() + (alpha * g * n).abs()
    else:
        x2 = x
    if pre:
        r2 = 1 / torch.sqrt((x2 * x2).sum(1, keepdim=True) / H + eps)
        res["h"] = x2 * r2 * w_pre
        res["h_size"] = (res.get("x_out_size", x.abs()) * r2 * w_pre.abs()).expand_as(x2)
    if not backward:
        return res
    d = torch.zeros_like(x2) if dx_out is None else dx_out.double()
    size = d.abs()
    if pre:
        xh, dh = x2 * r2, dh.double()
        u = dh * w_pre
        d = d + r2 * (u - xh * (u * xh).mean(1, keepdim=True))
        # x' is itself a sum: where x and the block's part cancel, its error is 2^-24 of the two, not of what is left
        xs = r2 * res.get("x_out_size", x.abs())
        size = size + r2 * (u.abs() + xs * (u.abs() * xs).mean(1, keepdim=True))
        res["dw_pre"], res["dw_pre_size"] = (dh * xh).sum(0), (dh.abs() * xs).sum(0)
    res["dx"], res["dx_size"] = d, size
    if y is not None:
        yh, v, vs = y * r, alpha * d * g * w_post, abs(alpha) * size * (g * w_post).abs()
        res["dy"], res["dy_size"] = v, vs
        if post:
            res["dy"] = r * (v - yh * (v * yh).mean(1, keepdim=True))
            res["dy_size"] = r * (vs + yh.abs() * (vs * yh.abs()).mean(1, keepdim=True))
            res["dw_post"], res["dw_post_size"] = (alpha * d * g * yh).sum(0), (abs(alpha) * size * (g * yh).abs()).sum(0)
        if gate is not None:
            t, s = alpha * d * n * slope, abs(alpha) * size * (n * slope).abs()
            res["dgate"], res["dgate_size"] = (t.sum(0), s.sum(0)) if gate.dim() == 1 else (t, s)
    return res


def policy(z, labels, old, ref, adv, tau, low, high, kl, row_grad=None):
    """loss, logp, dz, and how far rounding in 32 bits may move each: the log-probability by `moved` (a few units of the sum's and of
    the exponents' 2^-24), what hangs on it by its slope times that, a probability by 2e-5 of itself (exponents up to 128); one below 2^-126, FP32's smallest normal number,
    may be zero."""
    z = z.double()
    N, V = z.shape
    loss, logp, dz = torch.zeros(N, dtype=F64), torch.zeros(N, dtype=F64), torch.zeros(N, V, dtype=F64)
    loss_tol, logp_tol, dz_tol = torch.zeros(N, dtype=F64), torch.zeros(N, dtype=F64), torch.zeros(N, V, dtype=F64)
    z = z.cpu()
    for r in range(N):
        y = int(labels[r])
        if not 0 <= y < V:
            continue
        lp = torch.log_softmax(z[r] / tau, 0)
        logp[r] = lp[y]
        moved = 5e-6 + 2.0 ** -22 * abs(float(lp[y]))
        slope = bend = 0.0
        a = 0.0 if adv is None else float(adv[r])
        if a != 0.0:
            ratio = 1.0 if old is None else math.exp(float(lp[y]) - float(old[r]))
            loss[r] -= min(ratio * a, min(max(ratio, 1 - low), 1 + high) * a)
            if (ratio <= 1 + high) if a > 0 else (ratio >= 1 - low):
                slope -= a * ratio
                bend += abs(a) * ratio * (0.0 if old is None else 1.0)
        if ref is not None and kl != 0.0:
            k = float(ref[r]) - float(lp[y])
            loss[r] += kl * (math.exp(k) - k - 1)
            slope += kl * (1 - math.exp(k))
            bend += abs(kl) * math.exp(k)
        # the loss's slope: without old the ratio is 1 whatever logp is
        loss_tol[r] = (bend + abs(kl if ref is not None else 0.0)) * moved + 2.0 ** -23 * (abs(float(loss[r])) + abs(a))
        logp_tol[r] = moved
        g = (1.0 if row_grad is None else float(row_grad[r])) / tau
        p = torch.exp(lp)
        hot = torch.zeros(V, dtype=F64)
        hot[y] = 1.0
        dz[r] = g * slope * (hot - p)
        dz_tol[r] = abs(g) * ((bend * moved + 2.0 ** -22 * abs(slope)) * (hot - p).abs() + abs(slope) * (p * (2e-5 + moved) + 2.0 ** -126))
    return (loss, logp, dz), (loss_tol, logp_tol, dz_tol)


def clip(grads, scale, max_norm):
    """The outputs, and S, norm, coefficient, flag."""
    total = sum((float((t.double() * scale).square().sum()) for t in grads), 0.0)
    norm = math.sqrt(total) if total == total else math.nan
    coef = 1.0
    if max_norm > 0:
        coef = max_norm / (norm + 1e-6)
        coef = 1.0 if coef > 1.0 else coef
    return [t.double() * scale * coef for t in grads], [total, norm, coef, 0.0 if math.isfinite(norm) else 1.0]
