"""Embedding, block norms, policy loss and clipping as programs call them: waits that run out, captured and replayed, on several streams
and threads, queued behind each other, with offsets past 32 bits, and the arguments that are refused."""
import math
import threading

import pytest
import torch

import more_operators_ref as ref
from test_more_operators_gpu import BF16, F32, F64, assert_close, ctx, gen, half_step, policy_inputs, policy_case_outputs, randn, sd, spread_ids  # noqa: F401
from test_operators_waits_gpu import POLLS, out_of_patience

pytestmark = pytest.mark.gpu


def same(outs, want):
    def check():
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
    return check


# ---- waits that run out ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(400, 50000), (170, 72000), (6, 131072), (200, 35001)])
def test_policy_waits_that_run_out(ctx, sd, dtype, rows, vocab):
    a = policy_inputs(rows, vocab, dtype, seed=5)
    out = [torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(a["z"])]
    call = lambda: ctx.slidedp_policy_step(a["z"], a["labels"], a["old"], a["ref"], a["adv"], a["g"], *out, kl_weight=0.05)  # noqa: E731
    call()
    want = [x.clone() for x in out]
    for polls in POLLS:
        for x in out:
            x.fill_(7.0)
        out_of_patience(ctx, sd, polls, call, same(out, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H", [(3000, 4096), (2000, 1000), (900, 513), (700, 6400), (4000, 64)])
def test_norm_waits_that_run_out(ctx, sd, dtype, T, H):
    g = gen(T)
    x, y, gx, gh, gate = (randn(g, T, H, dtype=dtype) for _ in range(5))
    w = randn(g, H, dtype=dtype)
    fwd, bwd = [torch.empty_like(x) for _ in range(2)], [torch.empty_like(x) for _ in range(3)] + [torch.empty(H, device="cuda") for _ in range(2)]
    ws = torch.empty(ctx.slidedp_block_norm_workspace(x), dtype=torch.uint8, device="cuda")
    for call, out in ((lambda: ctx.slidedp_block_norm(x, y, w, gate, w, *fwd), fwd),
                      (lambda: ctx.slidedp_block_norm_backward(x, y, w, gate, w, gx, gh, *bwd, ws), bwd)):
        call()
        want = [t.clone() for t in out]
        for polls in POLLS:
            for t in out:
                t.fill_(7.0)
            out_of_patience(ctx, sd, polls, call, same(out, want))


# ---- all of them in one go -------------------------------------------------------------------------

class Pass:
    """Every operator once, on tensors of its own; `run` returns what it wrote."""

    def __init__(self, ctx, seed=0, T=700, H=512, V=33000):
        g = gen(seed)
        self.ctx = ctx
        self.ids = spread_ids(T, V, seed).to(torch.int32).cuda()
        self.table, self.dy = randn(g, V, H, dtype=BF16), randn(g, T, H, dtype=BF16)
        self.emb, self.d_table = torch.empty(T, H, dtype=BF16, device="cuda"), torch.empty(V, H, dtype=BF16, device="cuda")
        self.y, self.gx, self.gh = (randn(g, T, H, dtype=BF16) for _ in range(3))
        self.w, self.gate = randn(g, H, dtype=BF16), randn(g, H, dtype=BF16)
        self.norm = [torch.empty_like(self.y) for _ in range(4)] + [torch.empty(H, device="cuda") for _ in range(3)]
        self.policy = policy_inputs(40, 40000, BF16, seed)
        self.loss = [torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), torch.empty_like(self.policy["z"])]
        self.dz2 = torch.empty_like(self.policy["z"])
        self.grads = [randn(g, n) for n in (5000, 1, 70001)]
        self.clipped = [torch.empty(t.numel(), dtype=BF16, device="cuda") for t in self.grads]
        self.result = torch.empty(4, dtype=F64, device="cuda")
        ws = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.ws = [ws(ctx.slidedp_embedding_workspace(self.dy, self.d_table)), ws(ctx.slidedp_block_norm_workspace(self.y)),
                   ws(ctx.slidedp_clip_grad_norm_workspace(self.grads))]

    def outputs(self):
        return [self.emb, self.d_table, *self.norm, *self.loss, self.dz2, *self.clipped, self.result]

    def run(self, stream=None):
        c, p, n = self.ctx, self.policy, self.norm
        s = dict(stream=stream)
        c.slidedp_embedding(self.table, self.ids, self.emb, **s)
        c.slidedp_block_norm(self.emb, self.y, self.w, self.gate, self.w, n[0], n[1], **s)
        ins = (p["z"], p["labels"], p["old"], p["ref"], p["adv"])
        c.slidedp_policy_step(*ins, p["g"], *self.loss, kl_weight=0.1, **s)
        c.slidedp_policy_loss(*ins, self.loss[0], self.loss[1], kl_weight=0.1, **s)
        c.slidedp_policy_loss_backward(*ins, self.loss[1], p["g"], self.dz2, kl_weight=0.1, **s)
        c.slidedp_block_norm_backward(self.emb, self.y, self.w, self.gate, self.w, self.gx, self.gh, n[2], n[3], n[4], n[5], n[6], self.ws[1], **s)
        c.slidedp_embedding_backward(self.ids, n[2], self.d_table, self.ws[0], **s)
        c.slidedp_clip_grad_norm(self.grads, self.clipped, 0.5, self.result, self.ws[2], **s)
        return self.outputs()


def test_captured_and_replayed(ctx):
    a = Pass(ctx)
    want = [t.clone() for t in a.run()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(3):
        for t in a.outputs():
            t.fill_(math.nan)
        graph.replay()
        same(a.outputs(), want)()
    # what a replay reads is what is there then
    a.gx.mul_(0.5), a.policy["adv"].neg_(), a.grads[2].add_(1.0)
    want = [t.clone() for t in a.run()]
    for t in a.outputs():
        t.fill_(math.nan)
    graph.replay()
    same(a.outputs(), want)()


def test_two_graphs_side_by_side(ctx):
    passes = [Pass(ctx, seed) for seed in (1, 2)]
    wants = [[t.clone() for t in a.run()] for a in passes]
    torch.cuda.synchronize()
    graphs = []
    for a in passes:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            a.run()
        for t in a.outputs():
            t.fill_(math.nan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in passes]
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for a, want in zip(passes, wants):
        same(a.outputs(), want)()


def test_streams_and_threads_share_a_context(ctx):
    passes = [Pass(ctx, seed) for seed in (3, 4, 5)]
    wants = [[t.clone() for t in a.run()] for a in passes]
    for a in passes:
        for t in a.outputs():
            t.fill_(math.nan)
    torch.cuda.synchronize()
    errors = []

    def work(a):
        try:
            s = torch.cuda.Stream()
            for _ in range(6):
                a.run(s)
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(a,)) for a in passes]
    [t.start() for t in threads], [t.join() for t in threads]
    assert not errors
    for a, want in zip(passes, wants):
        same(a.outputs(), want)()


def test_each_call_sees_what_was_queued_before_it(ctx):
    """Calls whose kernels are set up while the ones before them end: chains of the same workspaces and buffers, again and again."""
    a = Pass(ctx, seed=6, T=64, H=256, V=600)
    want = [t.clone() for t in a.run()]
    for _ in range(30):
        a.run()
    same(a.outputs(), want)()
    x = randn(gen(7), 500, 256, dtype=BF16)
    w = torch.ones(256, dtype=BF16, device="cuda")
    one, two = torch.empty_like(x), torch.empty_like(x)
    chain, direct = x.clone(), x.clone()
    for _ in range(20):                       # each reads what the one before wrote
        ctx.slidedp_block_norm(chain, chain, w, None, w, one, two, residual_scale=0.1)
        chain, one = one, chain
    for _ in range(20):
        out, h = torch.empty_like(x), torch.empty_like(x)
        ctx.slidedp_block_norm(direct, direct, w, None, w, out, h, residual_scale=0.1)
        torch.cuda.synchronize()
        direct = out
    assert torch.equal(chain, direct)


# ---- offsets past 32 bits ----------------------------------------------------------------------------

def test_embedding_offsets_past_32_bits(ctx):
    V, H = 140000, 16384                      # 4.6 GB
    table = torch.zeros(V, H, dtype=BF16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 1, 131073, V], dtype=torch.int32, device="cuda")
    rows = randn(gen(1), 5, H, dtype=BF16)
    table[V - 1], table[131073] = rows[0], rows[1]
    out = torch.empty(5, H, dtype=BF16, device="cuda")
    ctx.slidedp_embedding(table, ids, out)
    assert torch.equal(out, torch.stack([rows[0], torch.zeros_like(rows[0]), rows[0], rows[1], torch.zeros_like(rows[0])]))
    table.fill_(3.0)
    ws = torch.empty(ctx.slidedp_embedding_workspace(rows, table), dtype=torch.uint8, device="cuda")
    ctx.slidedp_embedding_backward(ids, rows, table, ws)
    assert torch.equal(table[V - 1], (rows[0].float() + rows[2].float()).to(BF16)) and torch.equal(table[131073], rows[3]) and torch.equal(table[0], rows[1])
    mask = torch.ones(V, dtype=torch.bool, device="cuda")
    mask[[0, 131073, V - 1]] = False
    for part, keep in zip(table.split(20000), mask.split(20000)):
        assert not part[keep].any()


@pytest.mark.parametrize("off", [0, 1])
def test_block_norm_offsets_past_32_bits(ctx, off):
    T, H, stride = 600, 640, 4 << 20          # rows 4 M elements apart
    whole = torch.zeros(T * stride + 8, dtype=BF16, device="cuda")
    far = whole[off:].as_strided((T, H), (stride, 1))
    g = gen(2)
    far.copy_(randn(g, T, H, dtype=BF16))
    near, y, w = far.contiguous(), randn(g, T, H, dtype=BF16), randn(g, H, dtype=BF16)
    gx, gh = randn(g, T, H, dtype=BF16), randn(g, T, H, dtype=BF16)
    ws = torch.empty(ctx.slidedp_block_norm_workspace(near), dtype=torch.uint8, device="cuda")
    outs = []
    for x in (near, far):
        o = [torch.empty_like(near) for _ in range(4)]
        ctx.slidedp_block_norm(x, y, w, None, w, *o[:2])
        ctx.slidedp_block_norm_backward(x, y, w, None, w, gx, gh, *o[2:], None, None, None, ws)
        outs.append(o)
    for a, b in zip(*outs):
        # rows off the 16-byte grid are added up in another order
        assert torch.equal(a, b) if off == 0 else float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(a.float().abs().max())
    ctx.slidedp_block_norm(near, y, w, None, w, far, outs[0][1])
    assert float((far.float() - outs[0][0].float()).abs().max()) <= 2.0 ** -7 * float(far.float().abs().max())


@pytest.mark.parametrize("dtype,rows", [(BF16, 20), (F32, 10)])
def test_policy_offsets_past_32_bits(ctx, dtype, rows):
    V, stride = 40000, 1 << 28                # rows 268 M elements apart
    a = policy_inputs(rows, V, dtype, seed=3)
    want = policy_case_outputs(ctx, a)
    whole = torch.empty((rows - 1) * stride + V, dtype=dtype, device="cuda")
    far = whole.as_strided((rows, V), (stride, 1))
    far.copy_(a["z"])
    loss, logp = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ctx.slidedp_policy_step(far, a["labels"], a["old"], a["ref"], a["adv"], a["g"], loss, logp, far, clip_high=0.28, kl_weight=0.05)
    assert torch.equal(far, want[2]) and torch.equal(loss, want[0]) and torch.equal(logp, want[1])


def test_clip_offsets_past_32_bits(ctx):
    n = (1 << 31) + 4099
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[-3:] = torch.tensor([3.0, 4.0, 12.0], dtype=BF16)
    result = torch.empty(4, dtype=F64, device="cuda")
    ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace([g]), dtype=torch.uint8, device="cuda")
    ctx.slidedp_clip_grad_norm([g], [g], 6.5, result, ws)
    assert result[1].item() == 13.0
    assert g[-3:].tolist() == [1.5, 2.0, 6.0] and not g[:-3].any()


# ---- refusals ------------------------------------------------------------------------------------------

def refused(sd, status, call):
    with pytest.raises(sd.SlideDPError) as e:
        call()
    assert e.value.status == status


def test_outputs_over_inputs_are_refused(ctx, sd):
    z = torch.zeros(8, 100, device="cuda")
    ids, lab, f = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    bad = sd.ERR_INVALID_ARG
    refused(sd, bad, lambda: ctx.slidedp_embedding(z, ids, z))
    refused(sd, bad, lambda: ctx.slidedp_embedding_backward(ids, z, z, ws))
    refused(sd, sd.ERR_MISALIGNED, lambda: ctx.slidedp_embedding_backward(ids, z, torch.zeros(9, 100, device="cuda"), ws[1:]))
    o = torch.empty_like(z)
    refused(sd, bad, lambda: ctx.slidedp_block_norm(z, z, None, None, None, o, o))
    wide = torch.zeros(8, 200, device="cuda")
    refused(sd, bad, lambda: ctx.slidedp_block_norm(wide[:, :100], z, None, None, None, wide.view(-1)[:800].view(8, 100), o))
    refused(sd, bad, lambda: ctx.slidedp_block_norm_backward(z, o, None, None, None, None, z, o, o, None, None, None, ws))
    refused(sd, bad, lambda: ctx.slidedp_policy_step(wide[:, :100], lab, None, None, f, None, torch.empty(8, device="cuda"), torch.empty(8, device="cuda"),
                                                      wide.view(-1)[:800].view(8, 100)))
    refused(sd, bad, lambda: ctx.slidedp_policy_loss(z, lab, None, None, f, None, torch.empty(8, device="cuda")))       # a loss without a place
    res = torch.empty(4, dtype=F64, device="cuda")
    refused(sd, bad, lambda: ctx.slidedp_clip_grad_norm([f], [torch.empty(7, device="cuda")], 1.0, res, ws))
    refused(sd, bad, lambda: ctx.slidedp_clip_grad_norm([f], [f.view(torch.bfloat16)[:8]], 1.0, res, ws))


def test_arguments_that_are_refused(ctx, sd):
    z, lab, f = torch.zeros(8, 100, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    o, res = torch.empty_like(z), torch.empty(4, dtype=F64, device="cuda")
    ws, bad = torch.empty(1 << 24, dtype=torch.uint8, device="cuda"), sd.ERR_INVALID_ARG
    for kw in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=1e-40), dict(clip_low=-0.1), dict(clip_high=math.inf), dict(kl_weight=1e39)):
        refused(sd, bad, lambda: ctx.slidedp_policy_loss(z, lab, None, None, f, torch.empty(8, device="cuda"), torch.empty(8, device="cuda"), **kw))
    for kw in (dict(eps=-1.0), dict(residual_scale=math.nan), dict(eps=1e-50)):
        refused(sd, bad, lambda: ctx.slidedp_block_norm(z, z, None, None, None, o, None, **kw))
    refused(sd, bad, lambda: ctx.slidedp_block_norm(torch.zeros(2, 16385, device="cuda"), None, None, None, None, None, torch.zeros(2, 16385, device="cuda")))
    refused(sd, bad, lambda: ctx.slidedp_embedding(z, lab, o, scale=math.inf))
    refused(sd, bad, lambda: ctx.slidedp_clip_grad_norm([f], None, math.nan, res, ws))
    refused(sd, bad, lambda: ctx.slidedp_clip_grad_norm([f], None, 1.0, res, ws, scale=1e39))
    with pytest.raises(TypeError):
        ctx.slidedp_embedding(z.half(), lab, o.half())
    with pytest.raises(TypeError):
        ctx.slidedp_embedding(z, lab.long(), o)
    with pytest.raises(ValueError):
        ctx.slidedp_embedding(z, lab, o[:7])
    with pytest.raises(ValueError):
        ctx.slidedp_embedding(z, lab, torch.zeros(100, 8, device="cuda").T)
    with pytest.raises(ValueError):
        ctx.slidedp_embedding_backward(lab, o, z, ws[:10])
    with pytest.raises(TypeError):
        ctx.slidedp_block_norm(z, z.bfloat16(), None, None, None, o, None)
    with pytest.raises(ValueError):
        ctx.slidedp_block_norm(z, z, torch.zeros(99, device="cuda"), None, None, o, None)
    with pytest.raises(ValueError):
        ctx.slidedp_block_norm(z, z, None, torch.zeros(99, device="cuda"), None, o, None)
    with pytest.raises(TypeError):
        ctx.slidedp_policy_loss(z, lab.float(), None, None, f, f, f)
    with pytest.raises(TypeError):
        ctx.slidedp_clip_grad_norm([f.double()], None, 1.0, res, ws)
    with pytest.raises(ValueError):
        ctx.slidedp_clip_grad_norm([z.T], None, 1.0, res, ws)
    with pytest.raises(ValueError):
        ctx.slidedp_clip_grad_norm([f, f], [f], 1.0, res, ws)
    # subclasses and parameters are tensors
    p = torch.nn.Parameter(torch.ones(8, device="cuda"))
    ctx.slidedp_clip_grad_norm([p], None, 1.0, res, ws)
    assert abs(res[1].item() - math.sqrt(8)) < 1e-12


def test_tensors_of_another_gpu_are_refused(ctx, sd):
    z = torch.zeros(8, 100, device="cuda")
    ids = torch.zeros(8, dtype=torch.int32)
    with pytest.raises(TypeError):
        ctx.slidedp_embedding(z, ids, torch.empty_like(z))          # on the host
    with pytest.raises(TypeError):
        ctx.slidedp_block_norm(z, z, None, None, None, torch.empty(8, 100), None)
    with pytest.raises(TypeError):
        ctx.slidedp_clip_grad_norm([torch.zeros(4)], None, 1.0, torch.empty(4, dtype=F64, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))


def test_sums_of_the_weights_gradients_without_tokens(ctx):
    x = torch.empty(0, 64, device="cuda")
    dw = [torch.full((64,), 5.0, device="cuda") for _ in range(2)]
    ws = torch.empty(ctx.slidedp_block_norm_workspace(x), dtype=torch.uint8, device="cuda")
    ctx.slidedp_block_norm(x, x, None, None, None, torch.empty_like(x), torch.empty_like(x))
    ctx.slidedp_block_norm_backward(x, x, dw[0], None, dw[1], x, x, x, x, None, *dw, ws)
    assert not dw[0].any() and not dw[1].any()
    f = torch.empty(0, device="cuda")
    ctx.slidedp_policy_step(torch.empty(0, 10, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), f, f, f, f, f, f, torch.empty(0, 10, device="cuda"))
