"""The operators where their inputs or their surroundings are out of the ordinary: NaN and infinities that the backward pass
must keep in their document, offsets past 2^31 elements, head groups cut over a cluster, kernels queued behind the ones that
make their inputs, and calls from several threads.

Most comparisons are of bits: the same values by another route through the same kernel. The others use the tolerances of
test_operators_gpu.py.
"""
import math
import threading

import pytest
import torch

import operators_ref as ref
from test_operators_gpu import BF16, F32, attn_case, ctx, distill_inputs, gen, randn, sd, tolerance, assert_close  # noqa: F401

pytestmark = pytest.mark.gpu


def attention_pass(ctx, q, k, v, do, **kw):
    T, Hq, _ = q.shape
    out, lse = torch.empty_like(q), torch.empty(Hq, T, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
    ctx.slidedp_attention(q, k, v, out, lse, **kw)
    ctx.slidedp_attention_backward(q, k, v, out, lse, do, dq, dk, dv, ws, **kw)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_backward_keeps_nan_and_infinities_in_their_document(ctx, D, softcap):
    T, cu_list = 300, [0, 130, 205, 270]
    g = gen(D)
    q, do = randn(g, T, 4, D, dtype=BF16), randn(g, T, 4, D, dtype=BF16)
    k, v = randn(g, T, 2, D, dtype=BF16), randn(g, T, 2, D, dtype=BF16)
    kw = dict(cu_docs=torch.tensor(cu_list, dtype=torch.int32, device="cuda"), softcap=softcap)
    clean = attention_pass(ctx, q, k, v, do, **kw)
    ok = ref.visible(T, cu_list, None, True, "cuda")
    want = ref.attention(q, k, v, D ** -0.5, ok, softcap, None, do)
    for x in (q, k, v, do):
        x[150, 0], x[160, 1, 3], x[170, 1, 0] = math.nan, math.inf, -math.inf    # the second document
        x[280] = math.nan                                                       # padding
        x[290] = math.inf
    got = attention_pass(ctx, q, k, v, do, **kw)
    whole = torch.cat([torch.arange(130), torch.arange(205, 270)]).cuda()       # documents one and three
    for n in ("out", "dq", "dk", "dv"):
        assert not got[n][whole].isnan().any(), n
        assert torch.all(got[n][270:] == 0), n
        # rows redone one by one add in another order: the tolerance, not the bits
        assert_close(n, got[n][whole], want[n][whole], tolerance(want[n], BF16, want[n + "_bound"])[whole])
    if softcap:   # tanh has two forms, chosen by the largest score of 32 rows, whichever document they are of
        assert_close("lse", got["lse"][:, whole], want["lse"][:, whole], 2e-5 + 2e-6 * want["lse"][:, whole].abs())
    else:
        assert torch.equal(got["lse"][:, whole], clean["lse"][:, whole])
    assert torch.all(got["lse"][:, 270:] == -math.inf)
    assert got["dq"][150:205, 0].isnan().any() and got["dv"][150, 0].isnan().any()


@pytest.mark.parametrize("Hq,Hk,D,T", [(40, 8, 128, 300), (7, 1, 128, 140), (6, 2, 96, 257), (32, 1, 64, 100), (3, 3, 128, 400),
                                       (64, 8, 128, 513)])
def test_attention_groups_cut_over_a_cluster(ctx, Hq, Hk, D, T):
    attn_case(ctx, T, Hq, Hk, D, cu=[0, T // 3, T], seed=Hq + D)


@pytest.mark.parametrize("D,layout", [(128, "contiguous"), (128, "odd")])
def test_attention_offsets_past_32_bits(ctx, D, layout):
    """Three tokens 2^30 + 8 elements apart: the last one's offset does not fit 31 bits. 4.3 GB for each of two tensors."""
    T, H, step = 3, 2, 2 ** 30 + 8
    g = gen(1)
    off = 0 if layout == "contiguous" else 1
    q, k, v, do = (randn(g, T, H, D, dtype=BF16) for _ in range(4))
    want = attention_pass(ctx, q, k, v, do)
    far = torch.empty(2 * step + 8 * H * D, dtype=BF16, device="cuda")
    far_out = torch.zeros(2 * step + 8 * H * D, dtype=BF16, device="cuda")
    place = lambda buf, i: buf.as_strided((T, H, D), (step, D, 1), off + i * H * D)     # noqa: E731
    ins = [place(far, i) for i in range(4)]
    for x, y in zip(ins, (q, k, v, do)):
        x.copy_(y)
    out, dq, dk, dv = (place(far_out, i) for i in range(4))
    lse = torch.empty(H, T, device="cuda")
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
    ctx.slidedp_attention(ins[0], ins[1], ins[2], out, lse)
    ctx.slidedp_attention_backward(ins[0], ins[1], ins[2], out, lse, ins[3], dq, dk, dv, ws)
    got = dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    if layout == "contiguous":      # the same kernels
        for n in want:
            assert torch.equal(got[n], want[n]), n
    else:                           # the general ones
        full = ref.attention(q, k, v, D ** -0.5, ref.visible(T, None, None, True, "cuda"), 0.0, None, do)
        for n in ("out", "dq", "dk", "dv"):
            assert_close(n, got[n], full[n], tolerance(full[n], BF16, full[n + "_bound"]))


@pytest.mark.parametrize("off", [0, 1])
def test_qk_offsets_past_32_bits(ctx, off):
    T, H, D, step = 3, 5, 64, 2 ** 30 + 8
    g = gen(2)
    q, k, dq, dk = (randn(g, T, H, D, dtype=BF16) for _ in range(4))
    w = randn(g, D, dtype=BF16)
    angles = torch.arange(T, device="cuda")[:, None] * torch.logspace(0, -3, D // 2, device="cuda")
    table = torch.cat([angles.cos(), angles.sin()], 1)
    far = torch.zeros(2 * step + 8 * H * D + off, dtype=BF16, device="cuda")
    place = lambda i: far.as_strided((T, H, D), (step, D, 1), off + i * H * D)     # noqa: E731
    ws = torch.empty(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8, device="cuda")

    def both(q, k, dq, dk, out):
        dw = torch.empty(2, D, device="cuda")
        ctx.slidedp_qk_norm_rope(q, k, w, w, table, None, out[0], out[1])
        ctx.slidedp_qk_norm_rope_backward(q, k, w, w, table, None, dq, dk, out[2], out[3], dw[0], dw[1], ws)
        return [*(x.clone() for x in out), dw]
    near = torch.empty(4 * T * H * D + off, dtype=BF16, device="cuda")       # the same alignment, so the same kernel
    want = both(*(near.new_empty(T * H * D + off)[off:].view(T, H, D).copy_(x) for x in (q, k, dq, dk)),
                [near[off + i * T * H * D:off + (i + 1) * T * H * D].view(T, H, D) for i in range(4)])
    ins = [place(i).copy_(x) for i, x in enumerate((q, k, dq, dk))]
    got = both(*ins, [place(4 + i) for i in range(4)])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,rows", [(BF16, 18), (F32, 10)])
def test_distill_offsets_past_32_bits(ctx, dtype, rows):
    V, stride = 2000, 2 ** 27 + 8 if dtype == BF16 else 2 ** 28 + 8       # the last row starts past 2^31 elements
    assert (rows - 1) * stride > 2 ** 31
    g = gen(3)
    near = torch.zeros(rows, V + 8, dtype=dtype, device="cuda")[:, :V]
    near.copy_(randn(g, rows, V, scale=3.0))
    far = torch.empty((rows - 1) * stride + V, dtype=dtype, device="cuda").as_strided((rows, V), (stride, 1))
    far.copy_(near)
    ids = torch.randint(0, V, (rows, 9), generator=g, device="cuda", dtype=torch.int32)
    t, labels = randn(g, rows, 9), torch.arange(rows, dtype=torch.int32, device="cuda")
    res = []
    for z in (near, far):
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(2, rows, device="cuda")
        ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, temperature=1.5, w_teacher=0.7, w_label=0.3)
        loss2, lse2 = torch.empty_like(loss), torch.empty_like(lse)
        ctx.slidedp_distill_step(z, ids, t, labels, None, loss2, lse2, z, temperature=1.5, w_teacher=0.7, w_label=0.3)
        res.append((loss, lse, loss2, lse2, z.clone()))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_each_call_sees_what_was_queued_before_it(ctx):
    """Inputs, offsets and tables written just before the call, outputs overwritten just after it: the kernels may be set up
    early but not read or write early."""
    T, H, K, D = 700, 8, 2, 64
    g = gen(4)
    sets = []
    for i in range(3):
        q, do = randn(g, T, H, D, dtype=BF16), randn(g, T, H, D, dtype=BF16)
        k, v = randn(g, T, K, D, dtype=BF16), randn(g, T, K, D, dtype=BF16)
        cu = torch.tensor([0, 50 + 100 * i, 600 + i, T], dtype=torch.int32, device="cuda")
        sets.append((q, k, v, do, cu, randn(g, T, D // 2 * 2)))
    w = torch.ones(D, dtype=BF16, device="cuda")
    hold = [torch.empty_like(x) for x in sets[0]]
    ids = torch.randint(0, H * D, (T, 4), generator=g, device="cuda", dtype=torch.int32)
    t = randn(g, T, 4)
    bufs = None

    def run(s, wait):
        nonlocal bufs
        sync = torch.cuda.synchronize if wait else (lambda: None)
        for h, x in zip(hold, s):
            h.copy_(x)
        sync()
        q, k, v, do, cu, table = hold
        if bufs is None:
            bufs = [torch.empty_like(x) for x in (q, k, q, q, k, v, q, k)]
        qn, kn, out, dq, dk, dv, eq, ek = bufs
        lse, dw = torch.empty(H, T, device="cuda"), torch.empty(2, D, device="cuda")
        wa = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
        wq = torch.empty(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8, device="cuda")
        loss, l2 = torch.empty(T, device="cuda"), torch.empty(2, T, device="cuda")
        ctx.slidedp_qk_norm_rope(q, k, w, w, table, None, qn, kn)
        sync()
        ctx.slidedp_attention(qn, kn, v, out, lse, cu_docs=cu)
        sync()
        z = out.view(T, H * D)
        ctx.slidedp_distill_step(z, ids, t, None, None, loss, l2, do.view(T, H * D))
        sync()
        ctx.slidedp_attention_backward(qn, kn, v, out, lse, do, dq, dk, dv, wa, cu_docs=cu)
        sync()
        ctx.slidedp_qk_norm_rope_backward(q, k, w, w, table, None, dq, dk, eq, ek, dw[0], dw[1], wq)
        sync()
        res = [x.clone() for x in (*bufs, lse, dw, loss)]
        for x in bufs:
            x.fill_(math.nan)
        return res

    want = [run(s, True) for s in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [run(s, False) for s in sets]
        for a, b in zip(got, want):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_threads_share_a_context(ctx):
    T, D = 64, 64
    cases = []
    for i in range(4):
        g = gen(i)
        H = 2 + 2 * i
        cases.append([randn(g, T + i, h, D, dtype=BF16) for h in (H, 2, 2, H)])
    want = [attention_pass(ctx, *c) for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(60):
                got = attention_pass(ctx, *cases[i])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(got[n], want[i][n]) for n in got):
                    wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_captured_in_a_graph(ctx):
    g = gen(6)
    T, H, K, D = 300, 4, 2, 128
    q, k, v, do = (randn(g, T, h, D, dtype=BF16) for h in (H, K, K, H))
    want = attention_pass(ctx, q, k, v, do)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = attention_pass(ctx, q, k, v, do)
    for x in got.values():
        x.fill_(math.nan)
    graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_tensor_checks(ctx):
    class Named(torch.Tensor):
        pass

    T, H, D = 20, 2, 64
    q = randn(gen(7), T, H, D, dtype=BF16)
    out, lse = torch.empty_like(q), torch.empty(H, T, device="cuda")
    ctx.slidedp_attention(q, q, q, out, lse)
    for same in (torch.nn.Parameter(q, requires_grad=False), q.as_subclass(Named)):
        out2, lse2 = torch.empty_like(q), torch.empty_like(lse)
        ctx.slidedp_attention(same, q, q, out2, lse2)
        assert torch.equal(out2, out) and torch.equal(lse2, lse)
    call = lambda **kw: ctx.slidedp_attention(**{**dict(q=q, k=q, v=q, out=out, lse=lse), **kw})   # noqa: E731
    for bad in (dict(v=q.float()), dict(v=q.cpu()), dict(out=None), dict(lse=lse.double()), dict(v=[1]),
                dict(cu_docs=torch.tensor([0, T], device="cuda"))):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(v=q[:-1]), dict(out=q[:, :1]), dict(lse=lse[:, :-1]), dict(v=q.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(lse=torch.empty(T, H, device="cuda").T), dict(q=q[0])):
        with pytest.raises(ValueError):
            call(**bad)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau,wl", [(2.0, 0.5), (0.5, 0.5), (1.0, 0.5), (2.0, 0.0), (100.0, 0.5), (0.03, 0.25)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("V", [3001, 70000])
def test_distill_backward_of_masked_and_far_off_rows(ctx, dtype, tau, wl, in_place, V):
    """The gradient from the saved lse: rows whose lse is large, or beyond FP32, or says nothing of the row's sum."""
    N = 9
    z, ids, t, labels, gr = distill_inputs(N, V, 6, dtype, seed=29)
    z[0, 100:] = -math.inf
    z[1, 50:] = torch.finfo(dtype).min
    z[2] -= 20000.0
    z[3] = torch.finfo(dtype).min
    z[4] += 700.0
    z[5] = 3.0
    z[6] -= 127.0
    z[7, 2000] = 250.0
    z[8, 7:] = torch.finfo(dtype).min
    ids[:, :] = torch.arange(6, device="cuda", dtype=torch.int32)
    labels[:] = 3
    labels[5] = -1
    t[5, :] = -math.inf
    kw = dict(temperature=tau, w_teacher=0.5, w_label=wl)
    loss, lse = torch.empty(N, device="cuda"), torch.empty(2, N, device="cuda")
    _, _, want = ref.distill(z.cpu(), ids.cpu(), t.cpu(), labels.cpu(), tau, 0.5, wl, gr.cpu())
    # a row of one value throughout is a uniform distribution, which the reference's own log p = z / tau - lse does not resolve
    want[3] = gr[3].double().cpu() * (0.5 * tau + wl) / V
    for k in range(6):
        q = torch.softmax(t[3].double().cpu() / tau, 0)[k]
        want[3, k] -= float(gr[3]) * 0.5 * tau * float(q)
    want[3, 3] -= float(gr[3]) * wl
    ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, **kw)
    dz = z if in_place else torch.empty_like(z)
    ctx.slidedp_distill_loss_backward(z, ids, t, labels, lse, gr, dz, **kw)
    # as for the step, and for rows near zero 2^-24 of lse's size (at most 128) for the two roundings of it
    gmax = float(gr.abs().max()) * (0.5 * tau + wl)
    tol = (2.0 ** -8 * want.abs() if dtype == BF16 else 1e-5 * want.abs()) + (4e-6 + 128 * 2.0 ** -24) * gmax + 1e-30
    assert_close("gradient", dz.cpu(), want, tol)


def test_distill_factors_that_fp32_does_not_hold_are_refused(ctx, sd):
    z, ids, t, labels, _ = distill_inputs(3, 50, 4, F32, seed=1)
    loss, lse = torch.full((3,), 7.0, device="cuda"), torch.full((2, 3), 7.0, device="cuda")
    for bad in (dict(temperature=1e-39), dict(temperature=1e39), dict(temperature=1e-46), dict(w_teacher=1e39), dict(w_label=-1e39),
                dict(temperature=1e15, w_teacher=1e15)):
        with pytest.raises(sd.SlideDPError) as e:
            ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, **bad)
        assert e.value.status == sd.ERR_INVALID_ARG, bad
    assert torch.all(loss == 7.0) and torch.all(lse == 7.0)
    ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, temperature=1e-30)


@pytest.mark.parametrize("D", [64, 128, 132])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_gradients_of_scores_near_the_cap(ctx, D, sign):
    """Scores six to nine times the cap, whose derivative (1e-5 to 1e-7) is what the gradients of q and k consist of."""
    T, H, cap = 300, 2, 1.0
    g = gen(D)
    q = torch.full((T, H, D), sign, dtype=BF16, device="cuda")
    k = (1 + 0.1 * randn(g, T, 1, 1).clamp(-1.5, 1.5) + 0.01 * randn(g, T, 1, D)).to(BF16)
    v, do = randn(g, T, 1, D, dtype=BF16), randn(g, T, H, D, dtype=BF16)
    scale = 7.4 / D
    got = attention_pass(ctx, q, k, v, do, scale=scale, softcap=cap)
    want = ref.attention(q, k, v, scale, ref.visible(T, None, None, True, "cuda"), cap, None, do)
    for n in ("out", "dq", "dk", "dv"):
        assert_close(n, got[n], want[n], tolerance(want[n], BF16, want[n + "_bound"]))


def test_outputs_over_inputs_are_refused(ctx, sd):
    T, H, D = 140, 2, 64
    q, k, v, do = (randn(gen(i), T, H, D, dtype=BF16) for i in range(4))
    out, dq, dk, dv = (torch.full_like(q, 3.0) for _ in range(4))
    lse = torch.empty(H, T, device="cuda")
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")

    def refused(call, **kw):
        with pytest.raises(sd.SlideDPError) as e:
            call(**kw)
        assert e.value.status == sd.ERR_INVALID_ARG, kw
    before = [x.clone() for x in (q, k, v, do, out)]
    args = dict(q=q, k=k, v=v, out=out, lse=lse)
    for x in (q, k, v):
        refused(ctx.slidedp_attention, **{**args, "out": x})
    args.update(d_out=do, dq=dq, dk=dk, dv=dv, workspace=ws)
    for o in ("dq", "dk", "dv"):
        for x in (q, k, v, do):
            refused(ctx.slidedp_attention_backward, **{**args, o: x})
    for bad in (dict(dk=dq), dict(dv=dk), dict(dv=dq)):
        refused(ctx.slidedp_attention_backward, **{**args, **bad})
    # in place with other strides
    x = torch.full((T * H * D * 2,), 2.0, device="cuda")
    a, b = x[:T * H * D].view(T, H, D), x.view(T, 2 * H, D)[:, :H]
    y = torch.empty_like(a)
    refused(ctx.slidedp_qk_norm_rope, q=a, k=a, w_q=None, w_k=None, cos_sin=None, positions=None, q_out=b, k_out=y)
    refused(ctx.slidedp_qk_norm_rope_backward, q=y, k=y, w_q=None, w_k=None, cos_sin=None, positions=None, dq_out=a, dk_out=a,
            dq=y.clone(), dk=b, dw_q=None, dw_k=None, workspace=None)
    z = x.view(T, -1)
    ids, t, loss, l2 = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.zeros(T, 1, device="cuda"), torch.empty(T, device="cuda"), torch.empty(2, T, device="cuda")
    V = z.shape[1] // 2
    refused(ctx.slidedp_distill_step, logits=z[:, :V], teacher_ids=ids, teacher_logits=t, labels=None, row_grad=None, loss=loss, lse=l2,
            d_logits=x[:T * V].view(T, V))
    torch.cuda.synchronize()
    for now, then in zip((q, k, v, do, out), before):
        assert torch.equal(now, then)
    assert torch.all(x == 2.0)


def test_tensors_of_another_gpu_are_refused(sd):
    """The library would hand their addresses to kernels on the context's GPU. With one GPU at hand it is the context that is
    told another number; the checks come before the library, which still has the first."""
    T, H, D = 20, 2, 64
    q = randn(gen(7), T, H, D, dtype=BF16)
    a, b, lse = torch.full_like(q, 3.0), torch.full_like(q, 3.0), torch.full((H, T), 3.0, device="cuda")
    z, ids, t = randn(gen(3), 3, 500), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), randn(gen(4), 3, 2)
    loss, l2, dz = torch.full((3,), 3.0, device="cuda"), torch.full((2, 3), 3.0, device="cuda"), torch.full_like(z, 3.0)
    with sd.slidedp_create(0, 0) as ctx:
        ws = torch.empty(max(ctx.slidedp_attention_workspace(q, q), ctx.slidedp_qk_norm_rope_workspace(q, q)), dtype=torch.uint8, device="cuda")
        before = ctx.slidedp_kernel_launches()
        ctx.device = 1
        for call in (lambda: ctx.slidedp_attention(q, q, q, a, lse),
                     lambda: ctx.slidedp_attention_backward(q, q, q, q, lse, q, a, b, b, ws),
                     lambda: ctx.slidedp_qk_norm_rope(q, q, None, None, None, None, a, b),
                     lambda: ctx.slidedp_qk_norm_rope_backward(q, q, None, None, None, None, q, q, a, b, None, None, None),
                     lambda: ctx.slidedp_distill_loss(z, ids, t, None, loss, l2),
                     lambda: ctx.slidedp_distill_loss_backward(z, ids, t, None, l2, None, dz),
                     lambda: ctx.slidedp_distill_step(z, ids, t, None, None, loss, l2, dz)):
            with pytest.raises(ValueError, match="cuda:1"):
                call()
        assert ctx.slidedp_kernel_launches() == before
        ctx.device = 0
        ctx.slidedp_attention(q, q, q, a, lse)
    torch.cuda.synchronize()
    for x in (b, loss, l2, dz):
        assert torch.all(x == 3.0)


def test_the_default_stream_is_torchs_current_one_on_the_contexts_device(ctx, sd):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert sd._stream(None, ctx.device) == side.cuda_stream == sd._stream(None)
    assert sd._stream(None, ctx.device) == torch.cuda.current_stream().cuda_stream
