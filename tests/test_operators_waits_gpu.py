"""Waits inside the operators' kernels that run out: the kernel returns, the next call says SLIDEDP_ERR_TIMEOUT once, and the
context works as before. The waits are made to run out by a short limit on healthy launches; nothing hangs or fails on the GPU."""
import threading

import pytest
import torch

from test_operators_gpu import BF16, F32, ctx, distill_inputs, gen, randn, sd  # noqa: F401

pytestmark = pytest.mark.gpu

POLLS = [0, 1, 2, 3, 5, 9, 20]     # 0: every wait gives up; others: some do, and not the same ones in every warp


def out_of_patience(ctx, sd, polls, call, check):
    """Runs `call` with the limit, then without: an operator call reports a wait that ran out, once, and does nothing then."""
    ctx.slidedp_test_wait_polls(polls)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        ctx.slidedp_test_wait_polls(-1)
    reported = False
    try:
        call()
    except sd.SlideDPError as e:
        assert e.status == sd.ERR_TIMEOUT
        reported = True
    if polls == 0:
        assert reported
    call()
    torch.cuda.synchronize()
    check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(3, 40000), (8, 131072)])
def test_distill_waits_that_run_out(ctx, sd, dtype, rows, vocab):
    z, ids, t, labels, gr = distill_inputs(rows, vocab, 12, dtype, seed=5)
    loss, lse, dz = torch.empty(rows, device="cuda"), torch.empty(2, rows, device="cuda"), torch.empty_like(z)
    kw = dict(temperature=1.5, w_teacher=0.7, w_label=0.3)
    step = lambda: ctx.slidedp_distill_step(z, ids, t, labels, gr, loss, lse, dz, **kw)   # noqa: E731
    forward = lambda: ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, **kw)         # noqa: E731
    cases = []
    for call, n in ((step, 3), (forward, 2)):      # the two add up in other orders: each is compared with itself
        call()
        cases.append((call, [x.clone() for x in (loss, lse, dz)[:n]]))

    def same(want):
        def check():
            for a, b in zip((loss, lse, dz), want):
                assert torch.equal(a, b)
        return check
    for polls in POLLS:
        for call, want in cases:
            for x in (loss, lse, dz):
                x.fill_(7.0)
            out_of_patience(ctx, sd, polls, call, same(want))


@pytest.mark.parametrize("T,Hq,Hk,D,cu", [(900, 16, 4, 128, [0, 300, 310, 900]), (700, 32, 32, 64, [0, 700]), (200, 8, 1, 128, None)])
def test_attention_waits_that_run_out(ctx, sd, T, Hq, Hk, D, cu):
    g = gen(T)
    q, k, v, do = (randn(g, T, h, D, dtype=BF16) for h in (Hq, Hk, Hk, Hq))
    cu = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(Hq, T, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
    forward = lambda: ctx.slidedp_attention(q, k, v, out, lse, cu_docs=cu)                                        # noqa: E731
    backward = lambda: ctx.slidedp_attention_backward(q, k, v, *saved, do, dq, dk, dv, ws, cu_docs=cu)            # noqa: E731
    forward()
    saved = [out.clone(), lse.clone()]
    backward()
    want = [x.clone() for x in (dq, dk, dv)]

    def same(got, want):
        def check():
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        return check
    for polls in POLLS + [50, 200]:
        out_of_patience(ctx, sd, polls, forward, same((out, lse), saved))
        out_of_patience(ctx, sd, polls, backward, same((dq, dk, dv), want))


def give_up(ctx):
    """Leaves a wait that ran out behind, unreported."""
    q = randn(gen(1), 200, 2, 64, dtype=BF16)
    ctx.slidedp_test_wait_polls(0)
    ctx.slidedp_attention(q, q, q, torch.empty_like(q), torch.empty(2, 200, device="cuda"))
    ctx.slidedp_test_wait_polls(-1)
    torch.cuda.synchronize()


def test_every_operator_and_the_norm_report_a_wait_that_ran_out(sd):
    T, H, D = 40, 2, 64
    q = randn(gen(2), T, H, D, dtype=BF16)
    out, out2, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(H, T, device="cuda")
    dw, n = torch.empty(2, D, device="cuda"), q.numel()
    z, ids, t = randn(gen(3), 3, 500), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), randn(gen(4), 3, 2)
    loss, l2 = torch.empty(3, device="cuda"), torch.empty(2, 3, device="cuda")
    tiles = torch.empty(1, dtype=torch.float64, device="cuda")
    ctx = sd.slidedp_create(0, 0)
    ws = torch.empty(max(ctx.slidedp_attention_workspace(q, q), ctx.slidedp_qk_norm_rope_workspace(q, q)), dtype=torch.uint8, device="cuda")
    ctx.slidedp_attention(q, q, q, out, lse)
    ctx.slidedp_grad_norm([q], n, 1.0, True)
    ctx.slidedp_grad_norm_tiles([q], n, 1.0, tiles)
    want = ctx.slidedp_grad_norm_finish(1.0, fetch=True)
    calls = [lambda: ctx.slidedp_attention(q, q, q, out2, lse),
             lambda: ctx.slidedp_attention_backward(q, q, q, out, lse, q, out2, out2.clone(), out2.clone(), ws),
             lambda: ctx.slidedp_qk_norm_rope(q, q, None, None, None, None, out2, out2.clone()),
             lambda: ctx.slidedp_qk_norm_rope_backward(q, q, None, None, None, None, q, q, out2, out2.clone(), *dw, ws),
             lambda: ctx.slidedp_distill_loss(z, ids, t, None, loss, l2),
             lambda: ctx.slidedp_distill_loss_backward(z, ids, t, None, l2, None, z.clone()),
             lambda: ctx.slidedp_distill_step(z, ids, t, None, None, loss, l2, z.clone()),
             lambda: ctx.slidedp_grad_norm_finish(1.0, fetch=True),
             lambda: ctx.slidedp_grad_norm_finish_from(tiles, 1, 1.0, fetch=True)]
    for call in calls:
        for _ in range(2):
            give_up(ctx)
            ctx.slidedp_grad_norm_finish(1.0)              # without waiting there is nothing to tell yet
            with pytest.raises(sd.SlideDPError) as e:
                call()
            assert e.value.status == sd.ERR_TIMEOUT
            call()
    torch.cuda.synchronize()
    assert ctx.slidedp_grad_norm_finish(1.0, fetch=True) == want
    give_up(ctx)
    with pytest.raises(sd.SlideDPError) as e:
        ctx.slidedp_destroy()
    assert e.value.status == sd.ERR_TIMEOUT
    ctx.slidedp_destroy()                                 # it is gone


def test_threads_on_a_context_count_and_fail_exactly(sd):
    """Several threads in one context's operators: no launch is lost from the count, and an injected failure happens once."""
    ctx, threads, calls = sd.slidedp_create(0, 0), 8, 1500
    failed, statuses = [], []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            x = randn(gen(i), 1, 2, 8)
            y = torch.empty_like(x)
            for _ in range(calls):
                try:
                    ctx.slidedp_qk_norm_rope(x, x, None, None, None, None, y, y)
                except sd.SlideDPError as e:
                    failed.append(i)
                    statuses.append(e.status)
            torch.cuda.current_stream().synchronize()
    try:
        for nth in (0, threads * calls // 2):
            before = ctx.slidedp_kernel_launches()
            ctx.slidedp_test_fail_nth_call(nth)
            ts = [threading.Thread(target=work, args=(i,)) for i in range(threads)]
            for t in ts:
                t.start()
            for t in ts:
                t.join()
            assert statuses == ([sd.ERR_CUDA] if nth else [])
            assert ctx.slidedp_kernel_launches() - before == threads * calls - len(failed)
    finally:
        ctx.slidedp_destroy()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distilled_rows_whose_sums_did_not_come_are_nan(ctx, sd, dtype):
    """Not something that could pass for a result."""
    rows, vocab = 3, 40000       # cut over a cluster
    z, ids, t, labels, gr = distill_inputs(rows, vocab, 12, dtype, seed=6)
    loss, lse, dz = torch.zeros(rows, device="cuda"), torch.zeros(2, rows, device="cuda"), torch.zeros_like(z)
    for two in (0.0, 0.3):
        ctx.slidedp_test_wait_polls(0)
        ctx.slidedp_distill_step(z, ids, t, labels, None, loss, lse, dz, temperature=1.5, w_teacher=0.7, w_label=two)
        torch.cuda.synchronize()
        ctx.slidedp_test_wait_polls(-1)
        has = ((ids >= 0) & (ids < vocab)).any(1) | ((labels >= 0) & (labels < vocab) if two else False)
        assert has.any() and loss[has].isnan().all() and lse[0].isnan().all() and dz[has].isnan().all()
        with pytest.raises(sd.SlideDPError):
            ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse)
