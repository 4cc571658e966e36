"""GPU parity of embedding, block norms, policy loss and clipping with their definitions in 64 bits (tests/more_operators_ref.py).

Tolerances, derived before the first run. An output's own rounding: half a step, 2^-8 (BF16) or 2^-24 (FP32) of the value. Before it:
  * embedding: one product forward; a sum of n terms in FP32 is off by at most n 2^-24 of the sum of their absolute values, the
    product with the scale and the value added to by one rounding more each;
  * block norms: means of up to 16384 products in FP32, at most 32 per thread one after the other and 10 joins, below 42 * 2^-24 of their
    absolute values, square roots, a few products, an exponential (2 + |x| units): 1e-5 of the absolute terms that make up a value,
    and of the largest of its row where it is a difference from a mean over the row; a sum over tokens adds one 2^-24 per token;
  * policy loss: see more_operators_ref.policy;
  * clipping: sums in FP64; a factor and a product in FP32, 2^-24 each.
"""
import math

import pytest
import torch

import more_operators_ref as ref
from test_operators_gpu import assert_close, gen, randn

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module")
def sd():
    import paper_2609_34162_b200.slidedp as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    c = sd.slidedp_create(0, 0)
    yield c
    c.slidedp_destroy()


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


class Matrix:
    """An output matrix inside a larger allocation of a fixed pattern, to see stores outside it. `gap` elements between rows, `off`
    elements before the first."""

    def __init__(self, rows, cols, dtype, gap=0, off=0, fill=7.0):
        self.whole = torch.full((64 + off + rows * (cols + gap) + 64,), fill, dtype=dtype, device="cuda")
        self.view, self.fill = self.whole[64 + off:].as_strided((rows, cols), (cols + gap, 1)), fill

    def check(self, what):
        mark = torch.zeros_like(self.whole, dtype=torch.bool)
        mark.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(True)
        assert torch.all(self.whole[~mark] == self.fill), f"{what}: stores outside the output"


LAYOUTS = [(0, 0), (8, 0), (3, 1), (2, 2)]


# ---- embedding -----------------------------------------------------------------------------------

def embed_case(ctx, T, V, H, ids, dtype=BF16, grad=BF16, accumulate=False, layout=(0, 0), scale=1.3, seed=0, forward=True):
    g = gen(seed)
    gap, off = layout
    ids = torch.as_tensor(ids, dtype=torch.int32, device="cuda")
    if forward:
        table = Matrix(V, H, dtype, gap, off)
        table.view.copy_(randn(g, V, H, dtype=dtype))
        out = Matrix(T, H, dtype, gap, off)
        ctx.slidedp_embedding(table.view, ids, out.view, scale=scale)
        want = ref.embedding(table.view, ids, scale)
        assert_close("out", out.view, want, (half_step(dtype) + 2.0 ** -23) * want.abs())
        out.check("out")
    dy = Matrix(T, H, dtype, gap, off)
    dy.view.copy_(randn(g, T, H, dtype=dtype))
    dy.view[(ids < 0) | (ids >= V)] = math.nan            # absent rows are not read
    results = []
    for _ in range(2):
        dt = Matrix(V, H, grad, gap, off)
        if accumulate:
            dt.view.copy_(randn(gen(seed + 1), V, H, dtype=grad))
        before = dt.view.clone() if accumulate else None
        ws = torch.full((ctx.slidedp_embedding_workspace(dy.view, dt.view),), 255, dtype=torch.uint8, device="cuda")
        ctx.slidedp_embedding_backward(ids, dy.view, dt.view, ws, scale=scale, accumulate=accumulate)
        results.append(dt)
    want, size, count = ref.embedding_backward(ids, dy.view, V, scale, before)
    assert_close("d_table", dt.view, want, half_step(grad) * want.abs() + (count + 3) * 2.0 ** -24 * size)
    assert torch.equal(results[0].view, results[1].view)
    if accumulate:
        quiet = count[:, 0] == 0
        assert torch.equal(dt.view[quiet], before[quiet])
    dt.check("d_table")


def spread_ids(T, V, seed=0):
    """Frequencies as in texts, a few absent ones of every kind among them."""
    g = torch.Generator().manual_seed(seed)
    ids = (float(V + 1) ** torch.rand(T, generator=g, dtype=F64)).long().clamp(1, V) - 1
    odd = torch.tensor([-1, V, -2147483648, 2147483647])
    where = torch.rand(T, generator=g) < 0.05
    return torch.where(where, odd[torch.randint(0, 4, (T,), generator=g)], ids)


@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (1, 7, 64), (5, 3, 10), (33, 50, 136), (17, 511, 257), (16, 512, 8), (1025, 300, 250), (2049, 100000, 40),
                                   (4100, 1000, 96), (9000, 40, 1031)])
@pytest.mark.parametrize("dtype,grad", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
def test_embedding(ctx, T, V, H, dtype, grad):
    embed_case(ctx, T, V, H, spread_ids(T, V, seed=T), dtype, grad, accumulate=(T + H) % 2 == 0, seed=H)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_embedding_of_strided_and_unaligned_rows(ctx, dtype, layout):
    embed_case(ctx, 333, 77, 264, spread_ids(333, 77), dtype, dtype, layout=layout)
    embed_case(ctx, 333, 77, 262, spread_ids(333, 77), dtype, F32, accumulate=True, layout=layout)


@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_of_one_token_repeated_and_of_absent_ones(ctx, accumulate):
    how = dict(accumulate=accumulate, forward=False)
    embed_case(ctx, 3000, 9, 72, torch.full((3000,), 4), **how)                    # one sum over every piece
    embed_case(ctx, 200, 9, 72, torch.full((200,), -1), **how)
    embed_case(ctx, 64, 9, 72, torch.arange(64) // 16, **how)                      # ids begin and end with a piece
    embed_case(ctx, 64, 9, 72, (torch.arange(64) + 8) // 16, **how)                # each across an edge
    embed_case(ctx, 70, 9, 72, torch.tensor([8] * 35 + [0] * 35), **how)
    embed_case(ctx, 40000, 5, 24, torch.arange(40000) % 7, BF16, F32, **how)       # longer pieces, some tokens absent
    embed_case(ctx, 140000, 3, 8, torch.arange(140000) * 7 % 4, F32, F32, **how)


def test_embedding_without_tokens(ctx):
    d = torch.full((5, 16), 3.0, device="cuda", dtype=BF16)
    none, ids = torch.empty(0, 16, device="cuda", dtype=BF16), torch.empty(0, dtype=torch.int32, device="cuda")
    ws = torch.empty(ctx.slidedp_embedding_workspace(none, d), dtype=torch.uint8, device="cuda")
    ctx.slidedp_embedding(d, ids, none)
    ctx.slidedp_embedding_backward(ids, none, d, ws, accumulate=True)
    assert torch.all(d == 3.0)
    ctx.slidedp_embedding_backward(ids, none, d, ws)
    assert torch.all(d == 0.0)


def test_embedding_sums_follow_the_ids_order(ctx):
    """The sort is stable: the sum of one id's tokens does not depend on which other ids lie between them, piece by piece."""
    g = gen(3)
    dy = randn(g, 16, 64)
    ids = torch.tensor([1, 5, 1, 1, 9, 1, 0, 1, 1, 1, 3, 1, 1, 1, 1, 1], dtype=torch.int32, device="cuda")
    d = torch.empty(10, 64, device="cuda")
    ws = torch.empty(ctx.slidedp_embedding_workspace(dy, d), dtype=torch.uint8, device="cuda")
    ctx.slidedp_embedding_backward(ids, dy, d, ws)
    mine = dy[ids == 1]
    total = torch.zeros(64, device="cuda")
    for row in mine:                                       # one piece: its rows one after the other
        total = total + row
    assert torch.equal(d[1], total)


# ---- block norms ---------------------------------------------------------------------------------

def norm_case(ctx, T, H, dtype=BF16, post=True, pre=True, gate=None, sigmoid=False, with_y=True, weights=True, dx_out=True, layout=(0, 0), seed=0,
              alpha=0.6, eps=1e-6, x=None, y=None, sums=True):
    g = gen(seed)
    gap, off = layout

    def rows(t=None, fill=7.0):
        m = Matrix(T, H, dtype, gap, off, fill)
        if t is not None:
            m.view.copy_(t)
        return m

    x = rows(randn(g, T, H, dtype=dtype, scale=2.0) if x is None else x)
    y = rows(randn(g, T, H, dtype=dtype) if y is None else y) if with_y else None
    w = [1 + 0.2 * randn(g, H) for _ in range(2)]
    w_post, w_pre = (t.to(dtype) if weights else None for t in w)
    gv = None if gate is None else randn(g, H, dtype=dtype) if gate == 1 else rows(randn(g, T, H, dtype=dtype)).view
    how = dict(residual_scale=alpha, eps=eps, post_norm=post, gate_sigmoid=sigmoid)
    view = lambda m: None if m is None else m.view  # noqa: E731
    x_out, h = rows() if with_y else None, rows() if pre else None
    ctx.slidedp_block_norm(x.view, view(y), w_post if post else None, gv, w_pre, view(x_out), view(h), **how)
    gx, gh = randn(g, T, H, dtype=dtype) if dx_out else None, randn(g, T, H, dtype=dtype) if pre else None
    dx, dy = rows(), rows() if with_y else None
    dgate = None if gate is None else torch.empty(H, device="cuda") if gate == 1 else rows()
    dw_post, dw_pre = torch.empty(H, device="cuda") if with_y and post and sums else None, torch.empty(H, device="cuda") if pre and sums else None
    ws = torch.full((ctx.slidedp_block_norm_workspace(x.view),), 255, dtype=torch.uint8, device="cuda")
    ctx.slidedp_block_norm_backward(x.view, view(y), w_post if post else None, gv, w_pre, gx, gh, dx.view, view(dy),
                                    view(dgate) if isinstance(dgate, Matrix) else dgate, dw_post, dw_pre, ws, **how)
    want = ref.block_norm(x.view, view(y), w_post, gv, w_pre, alpha, eps, post, sigmoid, gx, gh, pre, backward=True)
    got = dict(x_out=x_out, h=h, dx=dx, dy=dy, dgate=dgate, dw_post=dw_post, dw_pre=dw_pre)
    for name, t in got.items():
        if t is None:
            continue
        out = t.view if isinstance(t, Matrix) else t
        size = want[name + "_size"].expand_as(want[name])
        if size.dim() == 2:                        # differences from a mean over the row
            tol = half_step(dtype) * want[name].abs() + 1e-5 * size + 1e-6 * size.amax(1, keepdim=True)
        else:
            tol = (1e-5 + T * 2.0 ** -24) * size
        assert_close(name, out, want[name], tol + 1e-37)
        if isinstance(t, Matrix):
            t.check(name)
    return got


@pytest.mark.parametrize("H", [1, 2, 31, 64, 100, 257, 1000, 2056, 4096, 5120, 8190, 8192, 12288, 16384])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_widths(ctx, H, dtype):
    norm_case(ctx, 37, H, dtype, seed=H)
    norm_case(ctx, 37, H, dtype, seed=H, gate=2, sigmoid=True)


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("gate,sigmoid", [(None, False), (1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("dtype,H", [(BF16, 384), (BF16, 130), (F32, 200)])
def test_block_norm_forms(ctx, dtype, H, gate, sigmoid, pre, post):
    norm_case(ctx, 50, H, dtype, post, pre, gate, sigmoid, seed=3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_without_block_weights_or_gradients(ctx, dtype):
    norm_case(ctx, 33, 520, dtype, post=False, with_y=False)
    norm_case(ctx, 33, 520, dtype, post=False, with_y=False, dx_out=False, weights=False)
    norm_case(ctx, 33, 520, dtype, weights=False)
    norm_case(ctx, 33, 520, dtype, dx_out=False, gate=1)
    norm_case(ctx, 33, 520, dtype, dx_out=False, pre=False)
    norm_case(ctx, 33, 520, dtype, sums=False)
    norm_case(ctx, 33, 520, dtype, alpha=0.0, gate=2)
    norm_case(ctx, 33, 520, dtype, alpha=-2.5, eps=0.0)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_of_strided_and_unaligned_rows(ctx, dtype, layout):
    norm_case(ctx, 21, 512, dtype, layout=layout, gate=2)
    norm_case(ctx, 21, 514, dtype, layout=layout, gate=1)
    norm_case(ctx, 21, 513, dtype, layout=layout)


@pytest.mark.parametrize("T,H", [(1, 4096), (2, 64), (3001, 96), (1537, 1025), (5000, 512)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_lengths(ctx, T, H, dtype):
    norm_case(ctx, T, H, dtype, gate=1, sigmoid=True, seed=T)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_of_zeros_and_of_large_values(ctx, dtype):
    T, H = 5, 300
    x, y = randn(gen(1), T, H, dtype=dtype), randn(gen(2), T, H, dtype=dtype)
    x[0], y[0], y[1] = 0.0, 0.0, 0.0
    x[2], y[3], x[4], y[4] = x[2] * 1e15, y[3] * 1e15, x[4] * 1e-15, y[4] * 1e-12
    norm_case(ctx, T, H, dtype, x=x, y=y)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_in_place(ctx, dtype):
    g = gen(5)
    T, H = 301, 768
    x, y, gx, gh = (randn(g, T, H, dtype=dtype) for _ in range(4))
    gate, w = randn(g, T, H, dtype=dtype), [randn(g, H, dtype=dtype) for _ in range(2)]
    new = lambda: torch.empty_like(x)  # noqa: E731
    x2, h, dx, dy, dgate = (new() for _ in range(5))
    ws = torch.empty(ctx.slidedp_block_norm_workspace(x), dtype=torch.uint8, device="cuda")
    ctx.slidedp_block_norm(x, y, w[0], gate, w[1], x2, h)
    ctx.slidedp_block_norm_backward(x, y, w[0], gate, w[1], gx, gh, dx, dy, dgate, None, None, ws)
    a, b = x.clone(), y.clone()
    ctx.slidedp_block_norm(a, b, w[0], gate, w[1], a, b)
    assert torch.equal(a, x2) and torch.equal(b, h)
    a, b, c = gx.clone(), gh.clone(), gate.clone()
    ctx.slidedp_block_norm_backward(x, y, w[0], c, w[1], a, b, a, b, c, None, None, ws)
    assert torch.equal(a, dx) and torch.equal(b, dy) and torch.equal(c, dgate)
    a, b = x.clone(), y.clone()
    ctx.slidedp_block_norm_backward(a, b, w[0], gate, w[1], gx, gh, a, b, dgate, None, None, ws)
    assert torch.equal(a, dx) and torch.equal(b, dy)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_of_wide_rows(ctx, dtype):
    """Rows that do not fit a ring: several for each block, every form, and written where they were read."""
    norm_case(ctx, 310, 8200, dtype)
    norm_case(ctx, 310, 8200, dtype, gate=1, sigmoid=True)
    norm_case(ctx, 310, 8193, dtype, gate=2, sigmoid=True, layout=(3, 1))
    norm_case(ctx, 601, 8190, dtype, gate=2, sigmoid=True)          # of these FP32 rows two blocks per SM
    norm_case(ctx, 150, 9002, dtype, gate=2, pre=False, weights=False)
    norm_case(ctx, 150, 9002, dtype, gate=1, post=False, layout=(2, 0))
    norm_case(ctx, 150, 9000, dtype, with_y=False, post=False, dx_out=False)
    norm_case(ctx, 150, 9000, dtype, sums=False, weights=False)
    norm_case(ctx, 150, 9000, dtype, post=False, pre=False)
    g = gen(8)
    T, H = 320, 8704
    x, y, gx, gh, gate = (randn(g, T, H, dtype=dtype) for _ in range(5))
    w = [randn(g, H, dtype=dtype) for _ in range(2)]
    x2, h, dx, dy, dgate = (torch.empty_like(x) for _ in range(5))
    ctx.slidedp_block_norm(x, y, w[0], gate, w[1], x2, h)
    a, b = x.clone(), y.clone()
    ctx.slidedp_block_norm(a, b, w[0], gate, w[1], a, b)
    assert torch.equal(a, x2) and torch.equal(b, h)
    ctx.slidedp_block_norm_backward(x, y, w[0], gate, w[1], gx, gh, dx, dy, dgate, None, None, None)
    for places in ((0, 1, 2), (1, 2, 0), (3, 4, 1), (2, 3, 4), (4, 0, 3)):
        ins = [t.clone() for t in (x, y, gate, gx, gh)]
        p, q, r = (ins[i] for i in places)
        ctx.slidedp_block_norm_backward(ins[0], ins[1], w[0], ins[2], w[1], ins[3], ins[4], p, q, r, None, None, None)
        assert torch.equal(p, dx) and torch.equal(q, dy) and torch.equal(r, dgate)


def test_block_norm_rows_do_not_touch_each_other(ctx):
    g = gen(6)
    T, H = 400, 512
    x, y, gx, gh = (randn(g, T, H, dtype=BF16) for _ in range(4))
    w = randn(g, H, dtype=BF16)
    ws = torch.empty(ctx.slidedp_block_norm_workspace(x), dtype=torch.uint8, device="cuda")

    def both():
        out = [torch.empty_like(x) for _ in range(4)]
        ctx.slidedp_block_norm(x, y, w, None, w, *out[:2])
        ctx.slidedp_block_norm_backward(x, y, w, None, w, gx, gh, *out[2:], None, None, None, ws)
        return out
    clean = both()
    x[7, 3], y[100, 0], gx[200, 5], gh[399, 511] = math.nan, math.inf, math.nan, -math.inf
    spoilt = both()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[7, 100, 200, 399]] = False
    for a, b in zip(clean, spoilt):
        assert torch.equal(a[keep], b[keep])
    assert spoilt[0][7, 3].isnan() and spoilt[1][7].isnan().all() and spoilt[0][100].isnan().any() and spoilt[2][200, 5].isnan() and spoilt[2][399].isnan().any()


# ---- policy loss ---------------------------------------------------------------------------------

def policy_inputs(N, V, dtype, seed=0, spread=2.5, absent=0.15, tau=1.0, edge=1e-3):
    g = gen(seed)
    z = randn(g, N, V, dtype=dtype, scale=spread)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    lp = torch.log_softmax(z.double() / tau, 1).gather(1, labels[:, None])[:, 0]
    moved = 0.3 * randn(g, N).double()
    for at in (0.8, 1.28):                        # no ratio near an edge of the clipped range
        moved = torch.where((moved - math.log(at)).abs() < edge, moved + 3 * edge, moved)
    odd = torch.tensor([-1, V, -100, 2147483647], device="cuda")
    where = torch.rand(N, generator=g, device="cuda") < absent
    labels = torch.where(where, odd[torch.arange(N, device="cuda") % 4], labels).to(torch.int32)
    return dict(z=z, labels=labels, old=(lp - moved).float(), ref=(lp + 0.5 * randn(g, N)).float(), adv=randn(g, N), g=randn(g, N))


def policy_case(ctx, a, tau=1.0, low=0.2, high=0.28, kl=0.05, layout=(0, 0), check=True):
    z, dtype = a["z"], a["z"].dtype
    N, V = z.shape
    gap, off = layout
    m = Matrix(N, V, dtype, gap, off)
    m.view.copy_(z)
    how = dict(temperature=tau, clip_low=low, clip_high=high, kl_weight=kl)
    ins = (m.view, a["labels"], a["old"], a["ref"], a["adv"])
    new = lambda: torch.full((N,), 9.0, device="cuda")  # noqa: E731
    loss, logp, loss2, logp2 = new(), new(), new(), new()
    ctx.slidedp_policy_loss(*ins, loss, logp, **how)
    dz, dz2 = Matrix(N, V, dtype, gap, off), Matrix(N, V, dtype, gap, off)
    ctx.slidedp_policy_loss_backward(*ins, logp, a["g"], dz.view, **how)
    ctx.slidedp_policy_step(*ins, a["g"], loss2, logp2, dz2.view, **how)
    dz.check("backward"), dz2.check("step")
    if check:
        (wl, wp, wz), (tl, tp, tz) = ref.policy(z, a["labels"], a["old"], a["ref"], a["adv"], tau, low, high, kl, a["g"])
        for l, p, d, what in ((loss, logp, dz.view, "two calls"), (loss2, logp2, dz2.view, "step")):
            assert_close(what + ": loss", l.cpu(), wl, tl + 1e-30)
            assert_close(what + ": logp", p.cpu(), wp, tp)
            # a gradient below the type's smallest normal number may be zero
            assert_close(what + ": dz", d.cpu(), wz, tz + half_step(dtype) * wz.abs() + 1e-37)
    in_place = m
    ctx.slidedp_policy_step(*ins, a["g"], loss, logp, in_place.view, **how)
    assert torch.equal(in_place.view, dz2.view) and torch.equal(loss, loss2) and torch.equal(logp, logp2)
    return loss2, logp2, dz2.view


@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (5, 7), (17, 31), (40, 1000), (9, 4099), (5, 32768), (3, 50257), (2, 131072), (300, 257)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy(ctx, N, V, dtype):
    policy_case(ctx, policy_inputs(N, V, dtype, seed=V), kl=0.05 if N % 2 else 0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [0.05, 0.7, 3.0])
def test_policy_temperatures(ctx, dtype, tau):
    policy_case(ctx, policy_inputs(24, 3001, dtype, seed=2, tau=tau), tau=tau)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_of_strided_and_unaligned_rows(ctx, dtype, layout):
    policy_case(ctx, policy_inputs(33, 2048, dtype), layout=layout)
    policy_case(ctx, policy_inputs(33, 2051, dtype), layout=layout)
    policy_case(ctx, policy_inputs(6, 40003, dtype), layout=layout)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_terms_left_out(ctx, dtype):
    a = policy_inputs(64, 777, dtype, seed=8)
    for names in (("old",), ("ref",), ("adv",), ("g",), ("old", "ref"), ("old", "adv"), ("old", "ref", "adv", "g")):
        policy_case(ctx, {**a, **dict.fromkeys(names)}, kl=0.1)
    lp, want, loss = (torch.empty(64, device="cuda") for _ in range(3))
    ctx.slidedp_policy_loss(a["z"], a["labels"], None, None, None, None, lp)
    ctx.slidedp_policy_loss(a["z"], a["labels"], a["old"], a["ref"], a["adv"], loss, want)
    assert torch.equal(lp, want)


def test_policy_on_the_edges_of_the_clipped_range(ctx):
    """Without old_logp the ratio is one: with ranges that end there it counts as inside. Far outside: no gradient on one side."""
    a = policy_inputs(32, 100, F32, absent=0.0)
    policy_case(ctx, {**a, "old": None, "ref": None}, low=0.0, high=0.0)
    lp = torch.log_softmax(a["z"].double(), 1).gather(1, a["labels"].long()[:, None])[:, 0]
    for far in (-3.0, 3.0):
        _, _, dz = policy_case(ctx, {**a, "old": (lp - far).float(), "ref": None})
        quiet = (a["adv"] > 0) if far > 0 else (a["adv"] < 0)
        assert not dz[quiet].any() and dz[~quiet].any(1).all()
    policy_case(ctx, {**a, "old": (lp - 1.0).float(), "ref": None}, low=5.0, high=1e6)          # a range that clips nothing
    policy_case(ctx, {**a, "adv": torch.zeros(32, device="cuda"), "old": torch.full((32,), -1e30, device="cuda")})


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_logits_far_from_zero_and_masked(ctx, dtype):
    a = policy_inputs(24, 600, dtype, seed=4)
    lowest = torch.finfo(dtype).min
    z = a["z"].float()
    z[0:6] += 3000.0
    z[6:12, ::3] = -math.inf
    z[12:18, 1::2] = lowest
    z = z.to(dtype)
    z[18] = 0.0
    keep = torch.where(torch.arange(24, device="cuda") < 18, (a["labels"].clamp(min=0) // 6 * 6 + 2).clamp(max=598), a["labels"])     # labels that are not masked
    a["labels"] = torch.where((a["labels"] >= 0) & (a["labels"] < 600), keep, a["labels"]).to(torch.int32)
    a["z"] = z
    lp = torch.log_softmax(z.double(), 1).gather(1, a["labels"].clamp(0, 599).long()[:, None])[:, 0]
    a["old"], a["ref"] = (lp + 0.1).float(), (lp - 0.3).float()
    policy_case(ctx, a)


@pytest.mark.parametrize("V", [300, 70000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_absent_rows_are_not_read_and_nan_stays_in_its_row(ctx, V, dtype):
    a = policy_inputs(40, V, dtype, seed=6, absent=0.0)
    a["labels"][::4] = -100
    clean = policy_case(ctx, a, check=False)
    z = a["z"].clone()
    z[::8] = math.nan
    z[5, 17], z[9, V - 1], z[13, 0] = math.nan, math.inf, math.nan
    spoilt = policy_case_outputs(ctx, {**a, "z": z})
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[5, 9, 13]] = False
    for c, s in zip(clean, spoilt):
        assert torch.equal(c[keep], s[keep]) and s[~keep].isnan().all()
    assert not spoilt[2][::4].any() and not spoilt[0][::4].any()


def policy_case_outputs(ctx, a, **how):
    N = len(a["z"])
    out = [torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(a["z"])]
    ctx.slidedp_policy_step(a["z"], a["labels"], a["old"], a["ref"], a["adv"], a["g"], *out, **{**dict(clip_high=0.28, kl_weight=0.05), **how})
    return out


def test_policy_rows_that_are_alike_give_alike_bits(ctx):
    """Whatever block or place a row has, and how often it is run."""
    for V, dtype in ((1000, BF16), (40001, BF16), (131072, BF16), (50257, F32)):
        a = policy_inputs(3, V, dtype, seed=1, absent=0.0)
        b = {k: v[torch.arange(700 if V < 50000 else 160) % 3].contiguous() for k, v in a.items()}
        if V % 8:                                  # other rows have another alignment: compare those that have the same
            step = 3 * 8
            first = policy_case_outputs(ctx, b)
            for t in first:
                assert torch.equal(t[:step], t[step:2 * step])
        else:
            for t in policy_case_outputs(ctx, b):
                assert torch.equal(t[:3], t[3:6]) and torch.equal(t[:3], t[-(len(t) % 3) - 3:][:3])


# ---- clipping ------------------------------------------------------------------------------------

def clip_case(ctx, sizes, src=F32, dst=BF16, scale=0.5, max_norm=1.0, spread=1.0, views=False, in_place=False, seed=0):
    g = gen(seed)
    types = [(src, dst)] if isinstance(src, torch.dtype) else list(zip(src, dst))
    kinds = [types[i % len(types)] for i in range(len(sizes))]
    if views:                       # odd offsets into one buffer per type
        flat = {d: torch.zeros(sum(sizes) + 3 * len(sizes) + 9, dtype=d, device="cuda") for d in (BF16, F32)}
        grads, outs, at = [], [], 1
        buffers = {d: torch.full_like(flat[d], 7.0) for d in (BF16, F32)}
        for n, (s, d) in zip(sizes, kinds):
            grads.append(flat[s][at:at + n])
            outs.append(buffers[d][at:at + n])
            at += n + n % 3
    else:
        grads = [torch.empty(n, dtype=s, device="cuda") for n, (s, _) in zip(sizes, kinds)]
        outs = [torch.empty(n, dtype=d, device="cuda") for n, (_, d) in zip(sizes, kinds)]
    for t in grads:
        t.copy_(randn(g, t.numel(), scale=spread))
    want, res = ref.clip([t.clone() for t in grads], scale, max_norm)
    if in_place:
        outs = grads
    result = torch.empty(4, dtype=F64, device="cuda")
    ws = torch.full((ctx.slidedp_clip_grad_norm_workspace(grads),), 255, dtype=torch.uint8, device="cuda")
    ctx.slidedp_clip_grad_norm(grads, outs, max_norm, result, ws, scale=scale)
    assert_close("result", result.cpu(), torch.tensor(res, dtype=F64), 1e-12 * torch.tensor(res, dtype=F64).abs())
    for i, (o, w) in enumerate(zip(outs, want)):
        assert_close(f"tensor {i}", o, w, (half_step(o.dtype) + 2.0 ** -23) * w.abs() + 1e-44)
    if views and not in_place:
        for d in (BF16, F32):
            mark = torch.zeros_like(buffers[d], dtype=torch.bool)
            for o in outs:
                if o.dtype == d:
                    mark[o.storage_offset():o.storage_offset() + o.numel()] = True
            assert torch.all(buffers[d][~mark] == 7.0)
    return grads, outs, result


ALL = ([F32, BF16, F32, BF16], [BF16, BF16, F32, F32])


@pytest.mark.parametrize("views", [False, True])
@pytest.mark.parametrize("sizes", [[1], [4096], [16385, 0, 3, 70001], [8, 1, 4096, 4097, 15, 16384, 99999, 7, 1], [0, 0], [1 << 20, 5, 1 << 19]])
@pytest.mark.parametrize("kinds", [(F32, BF16), (BF16, BF16), (F32, F32), (BF16, F32), ALL])
def test_clip(ctx, kinds, sizes, views):
    clip_case(ctx, sizes, *kinds, views=views)


@pytest.mark.parametrize("count", [63, 64, 65, 960, 961, 2500])
def test_clip_of_many_tensors(ctx, count):
    clip_case(ctx, [(i * 7919) % 3001 for i in range(count)], *ALL, views=count % 2 == 1)


def test_clip_in_place_and_without_need(ctx):
    for src in (BF16, F32):
        clip_case(ctx, [5000, 3, 70000], src, src, in_place=True)
        clip_case(ctx, [5000, 3, 70000], src, src, views=True, in_place=True)
        clip_case(ctx, [5000, 3, 70000], src, src, max_norm=0.0, in_place=True)
        clip_case(ctx, [5000, 3, 70000], src, src, max_norm=1e9)
        grads, _, _ = clip_case(ctx, [5000, 33], src, src, scale=1.0, max_norm=1e9, in_place=True)
    clip_case(ctx, [100000] * 20, F32, BF16, max_norm=0.0, scale=-0.3)
    clip_case(ctx, [10000], F32, F32, spread=1e30)               # squares beyond FP32
    clip_case(ctx, [10000], F32, F32, spread=1e-30)


def test_clip_none_at_all(ctx):
    result = torch.full((4,), 5.0, dtype=F64, device="cuda")
    ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace([]), dtype=torch.uint8, device="cuda")
    ctx.slidedp_clip_grad_norm([], [], 1.0, result, ws)
    assert result.tolist() == [0.0, 0.0, 1.0, 0.0]
    g = [randn(gen(1), 1000)]
    ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace(g), dtype=torch.uint8, device="cuda")
    before = g[0].clone()
    ctx.slidedp_clip_grad_norm(g, None, 1e-3, result, ws)
    assert torch.equal(g[0], before) and abs(result[1].item() - before.double().norm().item()) < 1e-9


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_clip_with_a_norm_that_is_not_finite(ctx, bad):
    g = [randn(gen(1), 5000), randn(gen(2), 70000)]
    g[1][69999] = bad
    outs = [torch.empty(t.numel(), dtype=BF16, device="cuda") for t in g]
    result = torch.empty(4, dtype=F64, device="cuda")
    ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace(g), dtype=torch.uint8, device="cuda")
    ctx.slidedp_clip_grad_norm(g, outs, 1.0, result, ws)
    assert result[3].item() == 1.0
    if math.isnan(bad):
        assert result[2].isnan() and all(o.isnan().all() for o in outs)
    else:
        assert result[2].item() == 0.0 and not outs[0].any() and outs[1][69999].isnan() and not outs[1][:69999].any()


def test_clip_is_the_norm_of_the_flat_path(ctx):
    """The same numbers as slidedp_grad_norm of the concatenation."""
    g = gen(9)
    parts = [randn(g, n, dtype=BF16, scale=1e-3) for n in (16384, 16384 * 3, 16384 * 2 + 777)]
    flat = torch.cat(parts)
    ctx.slidedp_grad_norm([flat], flat.numel(), 0.5)
    norm, coef = ctx.slidedp_grad_norm_finish(0.1, fetch=True)
    _, _, result = None, None, torch.empty(4, dtype=F64, device="cuda")
    ws = torch.empty(ctx.slidedp_clip_grad_norm_workspace(parts), dtype=torch.uint8, device="cuda")
    ctx.slidedp_clip_grad_norm(parts, None, 0.1, result, ws, scale=0.5)
    assert abs(result[1].item() - norm) <= 1e-12 * norm and abs(result[2].item() - coef) <= 1e-12 * coef


@pytest.mark.parametrize("V", [9, 1000, 20000, 70000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_rows_of_the_lowest_value(ctx, V, dtype):
    """All logits masked with the type's lowest value: as likely as each other. Some of them: not at all. Very large ones beside them."""
    a = policy_inputs(8, V, dtype, absent=0.0)
    lowest = torch.finfo(dtype).min
    z = a["z"].clone()
    z[0], z[1], z[2] = lowest, lowest, -lowest
    z[1, ::2] = -math.inf
    z[2, 1::3] = 1.0
    z[3], z[3, 5:8] = 1e30, 2e30
    z[4], z[4, 2] = lowest, 0.0
    a["z"], a["labels"] = z, torch.tensor([3, 5, 0, 6, 2, 1, 2, 3], dtype=torch.int32, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, a["labels"].long()[:, None])[:, 0]
    a["old"], a["ref"] = (lp + 0.1).float(), (lp - 0.3).float()
    for tau in (1.0, 0.6):
        policy_case(ctx, a, tau=tau, kl=0.05 if tau == 1.0 else 0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_rows_at_the_limits_of_their_kernels(ctx, dtype):
    """Rows that just fit what a warp, a block or the ring holds, and rows one chunk longer, aligned and not."""
    per = 16 // dtype.itemsize
    for chunks in (128, 256, 512, 768, 1024, 1536, 2048, 2560, 4096, 8704):
        for V in (chunks * per, chunks * per + 1):
            a = policy_inputs(3, V, dtype, seed=chunks)
            policy_case(ctx, a)
            if chunks in (128, 2048, 4096):
                policy_case(ctx, a, layout=(1, 1))
