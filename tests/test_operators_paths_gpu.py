"""The operators at sizes where their kernels work as they do on training batches: blocks that take over several tiles, rings
that wrap, rows cut so that they stay in L2. And a bound on whole rows of the gradients, which a single pair that is masked
wrongly breaks where the elementwise bound of several hundred roundings does not."""
import math

import pytest
import torch

import operators_ref as ref
from test_operators_gpu import BF16, F32, assert_close, attn_case, ctx, distill_inputs, gen, qk_inputs, randn, sd, tolerance  # noqa: F401

pytestmark = pytest.mark.gpu


def row_bounds(a, cu, prefix, causal, softcap, slopes, scale):
    """For each row of out, dq, dk and dv how far its error may reach, in the 2-norm over the head's values.

    Probabilities and score gradients are rounded to BF16: relative errors e, independent, |e| <= u = 2^-8, variance at most
    u^2 / 3, each of which moves a row by e times a partner's vector. Their sum is at most the sum of the lengths, and with
    many partners near its standard deviation: six of them are allowed. The saved out is rounded as well and moves delta, the
    same for all partners of a query. Then each output is rounded (u of the row), and FP32 has 1e-5 of the tensor's scale.

    And for the whole tensor the expected square of the error: the variances, and 1e-5 of each row's terms for FP32."""
    q, k, v, do = (a[n].double() for n in ("q", "k", "v", "do"))
    T, Hq, D = q.shape
    G, u = Hq // k.shape[1], 2.0 ** -8
    ok = ref.visible(T, cu, prefix, causal, "cuda")
    dist = (torch.arange(T, device="cuda")[:, None] - torch.arange(T, device="cuda")[None, :]).abs().double()
    var = {n: torch.zeros(a["want"][n].shape[:2], dtype=torch.float64, device="cuda") for n in ("out", "dq", "dk", "dv")}
    hard = {n: torch.zeros_like(x) for n, x in var.items()}
    own = {n: torch.zeros_like(x) for n, x in var.items()}      # from delta
    for h in range(Hq):
        kk, vv, hk = k[:, h // G], v[:, h // G], h // G
        s = q[:, h] @ kk.T * scale
        grad = torch.ones_like(s)
        if softcap:
            th = torch.tanh(s / softcap)
            s, grad = softcap * th, 1 - th * th
        if slopes is not None:
            s = s - float(slopes[h]) * dist
        some = ok.any(1)
        L = torch.where(some, torch.logsumexp(torch.where(ok, s, -math.inf), 1), 0.0)
        p = torch.where(ok, torch.exp(s - L[:, None]), 0.0)
        out, g = p @ vv, do[:, h]
        dp = g @ vv.T
        ds = p * (dp - (p * dp).sum(1, keepdim=True)) * grad * scale
        n2 = lambda x: (x * x).sum(1)  # noqa: E731
        var["out"][:, h] = u * u / 3 * (p * p @ n2(vv))
        hard["out"][:, h] = u * (p @ n2(vv).sqrt())
        delta = (g * g * (u * u / 3 * (out * out + p * p @ (vv * vv)))).sum(1)          # variance of delta
        var["dq"][:, h] = u * u / 3 * (ds * ds @ n2(kk))
        hard["dq"][:, h] = u * (ds.abs() @ n2(kk).sqrt())
        own["dq"][:, h] = delta * n2((p * grad * scale) @ kk)
        var["dk"][:, hk] += u * u / 3 * (ds * ds).T @ n2(q[:, h])
        hard["dk"][:, hk] += u * ds.abs().T @ n2(q[:, h]).sqrt()
        own["dk"][:, hk] += (p * grad * scale).square().T @ (delta * n2(q[:, h]))
        var["dv"][:, hk] += u * u / 3 * (p * p).T @ n2(g)
        hard["dv"][:, hk] += u * p.T @ n2(g).sqrt()
    res = {}
    for n in var:
        w = a["want"][n]
        rounded = w.square().sum(2)
        rows = (torch.minimum(hard[n], 6 * var[n].sqrt()) + 6 * own[n].sqrt() + u * rounded.sqrt()
                + 1e-5 * float(w.abs().max()) * math.sqrt(D) + 1e-30)
        res[n] = rows, float((var[n] + own[n] + u * u / 3 * rounded + (1e-5 / u * hard[n]) ** 2).sum()) + 1e-30
    return res


def case(ctx, T, Hq, Hk, D, cu=None, prefix=None, causal=True, softcap=0.0, bias=False, seed=0, spread=1.0):
    a = attn_case(ctx, T, Hq, Hk, D, cu=cu, prefix=prefix, causal=causal, softcap=softcap, bias=bias, seed=seed, spread=spread)
    bounds = row_bounds(a, cu, prefix, causal, softcap, a["kw"]["slopes"], D ** -0.5)
    for n, (rows, total) in bounds.items():
        err = (a[n].double() - a["want"][n]).square().sum(2)
        bad = ~(err.sqrt() <= rows)
        assert not bad.any(), f"{n}: {int(bad.sum())} rows, worst {float((err.sqrt() / rows).max()):.2f} of the bound"
        # the sum of thousands of independent squares is near what is expected: twice that is allowed
        assert float(err.sum()) <= 2 * total, f"{n}: {float(err.sum()) / total:.2f} of the expected square of the error"


FORMS = [dict(), dict(bias=True), dict(softcap=30.0), dict(softcap=5.0, bias=True, spread=1.5)]
IDS = ["plain", "bias", "cap", "cap_bias"]


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("D", [64, 128])
def test_blocks_that_take_over_tiles_of_keys(ctx, D, form):
    """352 tiles of keys and of queries, 192 items of the forward pass, for 148 SMs and nothing shared by a cluster; short and
    long documents, tiles without any."""
    case(ctx, 1300, 32, 32, D, cu=[10, 20, 400, 401, 530, 1010], seed=D, **form)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_groups_of_heads_in_many_tiles_of_keys(ctx, form):
    """320 tiles of keys, each walked for both heads of its group by one block."""
    case(ctx, 2500, 32, 16, 96, cu=[0, 700, 1800, 2490], prefix=[100, 0, 300], seed=5, **form)


@pytest.mark.parametrize("Hq,Hk,D", [(32, 32, 128), (20, 20, 40)])
def test_long_walks_in_both_directions(ctx, Hq, Hk, D):
    case(ctx, 2100, Hq, Hk, D, cu=[0, 2000, 2100], causal=False, seed=9)


@pytest.mark.parametrize("T,Hq,Hk", [(1531, 4, 1), (513, 16, 8), (257, 2, 2)])
@pytest.mark.parametrize("D", [64, 128, 136])
def test_rows_of_every_result(ctx, T, Hq, Hk, D):
    case(ctx, T, Hq, Hk, D, cu=[0, T // 3, T - 20], seed=T)


# ---- norm and rotation: more tasks than the grid takes at once -----------------------------------------

@pytest.mark.parametrize("T,Hq,Hk,D,rope,interleaved,dtype,layout", [
    (5003, 9, 2, 128, 128, False, BF16, "contiguous"),      # 1250 blocks of tasks for 592 (forward) and 444 (backward)
    (5003, 9, 2, 128, 64, True, BF16, "padded"),
    (3001, 7, 3, 80, 48, True, F32, "contiguous"),
    (3001, 5, 5, 128, 128, False, F32, "contiguous"),
    (9000, 3, 6, 64, 64, False, BF16, "contiguous"),
    (2500, 4, 4, 256, 256, True, BF16, "contiguous"),
    (4001, 5, 2, 96, 96, False, BF16, "padded"),
    (20011, 1, 0, 24, 8, False, BF16, "contiguous"),
    (2003, 3, 1, 33, 10, True, F32, "odd"),
])
def test_norm_in_several_rounds_of_the_grid(ctx, T, Hq, Hk, D, rope, interleaved, dtype, layout):
    q, k, gq, gk, wq, wk, cs, pos = qk_inputs(T, Hq, Hk, D, rope, dtype, layout, seed=3)
    yq, yk, dq, dk = (torch.full((T, h, D), math.nan, dtype=dtype, device="cuda") for h in (Hq, Hk, Hq, Hk))
    dwq, dwk = (torch.full((D,), 9.0, device="cuda") for _ in range(2))
    kw = dict(eps=1e-5, interleaved=interleaved)
    ws = torch.empty(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8, device="cuda")
    ctx.slidedp_qk_norm_rope(q, k, wq, wk, cs, pos, yq, yk, **kw)
    ctx.slidedp_qk_norm_rope_backward(q, k, wq, wk, cs, pos, gq, gk, dq, dk, dwq, dwk, ws, **kw)
    for x, w, gy, y, dx, dw, what in ((q, wq, gq, yq, dq, dwq, "q"), (k, wk, gk, yk, dk, dwk, "k")):
        want = ref.qk_forward(x, w, cs, pos, 1e-5, interleaved)
        assert_close("y of " + what, y, want, tolerance(want, dtype))
        wdx, wdw = ref.qk_backward(x, w, cs, pos, 1e-5, interleaved, gy)
        assert_close("dx of " + what, dx, wdx, tolerance(wdx, dtype))
        assert_close("dw of " + what, dw, wdw, 1e-5 * max(1.0, math.sqrt(T * max(x.shape[1], 1))) * 4)


# ---- distillation: many long rows ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,tau,wt,wl,labelled", [
    (600, 131072, 2.0, 1.0, 0.0, False), (600, 131072, 1.5, 0.7, 0.3, True), (600, 131072, 1.0, 0.0, 1.0, True),
    (700, 30011, 2.0, 0.5, 0.5, True), (2000, 8000, 1.0, 1.0, 0.0, False)])
def test_distillation_of_many_long_rows(ctx, dtype, rows, vocab, tau, wt, wl, labelled):
    """A sample of the rows against the definition; with and without a second softmax, each unroll, rows in one block or cut."""
    z, ids, t, labels, gr = distill_inputs(rows, vocab, 20, dtype, seed=rows + vocab)
    labels = labels if labelled else None
    kw = dict(temperature=tau, w_teacher=wt, w_label=wl)
    new = lambda *s: torch.full(s, 9.0, device="cuda")  # noqa: E731
    loss, lse, loss2, lse2, dz, dz2 = new(rows), new(2, rows), new(rows), new(2, rows), torch.empty_like(z), torch.empty_like(z)
    ctx.slidedp_distill_step(z, ids, t, labels, gr, loss, lse, dz, **kw)
    ctx.slidedp_distill_loss(z, ids, t, labels, loss2, lse2, **kw)
    ctx.slidedp_distill_loss_backward(z, ids, t, labels, lse2, gr, dz2, **kw)
    pick = torch.tensor(sorted({0, 1, 3, 4, rows // 3, rows // 2, rows - 1, *range(7, rows, 97)}), device="cuda")
    at = lambda x: None if x is None else x[pick].cpu()  # noqa: E731
    wloss, wlse, wdz = ref.distill(at(z), at(ids), at(t), at(labels), tau, wt, wl, at(gr))
    zmax, gmax = float(z[pick].float().abs().max()), float(gr.abs().max())
    # the tolerances of the small sizes; a row's FP32 sum of `vocab` terms adds 2^-24 sqrt(vocab) at most
    ltol = 1e-6 * (1 + wt * tau * tau * (zmax / tau + 12) + wl * (zmax + 12)) * 4
    gtol = (2.0 ** -8 * wdz.abs() if dtype == BF16 else 2e-5 * wdz.abs()) + 4e-6 * gmax * (wt * tau + wl) + 1e-30
    for l, s, d in ((loss, lse, dz), (loss2, lse2, dz2)):
        assert_close("loss", at(l), wloss, ltol)
        assert_close("lse", s[:, pick].cpu(), wlse, 1e-6 * (zmax / tau + zmax + 12))
        assert_close("gradient", at(d), wdz, gtol)
    # and every row: its gradient's sum over the vocabulary is zero but for the roundings (each of at most 2^-8 of its size),
    # and nothing is left unwritten
    for d in (dz, dz2):
        total, size = d.double().sum(1), d.double().abs().sum(1)
        assert torch.all(total.abs() <= (2.0 ** -8 if dtype == BF16 else 1e-5) * size + 1e-5), "sum of a row"
