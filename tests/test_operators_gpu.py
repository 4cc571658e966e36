"""GPU parity of the fine-tuning operators with their definitions in 64 bits (tests/operators_ref.py).

Tolerances, from the arithmetic that the header promises (u = 2^-8 is half a BF16 ulp, relative: eight
significant bits):
  * a BF16 output of FP32 arithmetic: u |y| for its rounding + 1e-5 of the tensor's scale for the
    FP32 sums and exponentials before it; an FP32 output: 1e-5 of its scale;
  * attention multiplies probabilities and score gradients as BF16, so an output also moves by up to
    u times the sum of the absolute terms (plus what the rounded saved `out` does to the gradients); the
    reference returns that bound element by element.
"""
import math

import pytest
import torch

import operators_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN_WORDS = 64     # guard elements around every output


@pytest.fixture(scope="module")
def sd():
    import paper_2609_34162_b200.slidedp as sd
    return sd


@pytest.fixture(scope="module")
def ctx(sd):
    c = sd.slidedp_create(0, 0)
    yield c
    c.slidedp_destroy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


class Guarded:
    """An output view inside a larger allocation of a fixed pattern, to see stores outside it."""

    def __init__(self, T, H, D, dtype, layout="contiguous"):
        self.layout = layout
        pad = {"contiguous": 0, "padded": 8, "odd": 3}[layout]       # elements between heads' rows
        row = H * (D + pad) + pad
        off = NAN_WORDS if layout != "odd" else NAN_WORDS + 1
        self.whole = torch.full((off + T * row + NAN_WORDS,), 7.0, dtype=dtype, device="cuda")
        self.view = self.whole[off:off + T * row].view(T, row)[:, :H * (D + pad)].view(T, H, D + pad)[..., :D]

    def check(self, what):
        seen = self.whole.clone()
        mark = torch.zeros_like(self.whole, dtype=torch.bool)
        mark.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(True)
        assert torch.all(seen[~mark] == 7.0), f"{what}: stores outside the output"


def assert_close(what, got, want, tol):
    got, want = got.double(), want.to(got.device).double()
    assert got.shape == want.shape, what
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got - want).abs() <= tol)
    if bad.any():
        i = int(bad.flatten().nonzero()[0])
        worst = float(((got - want).abs() / tol.clamp(min=1e-300) if torch.is_tensor(tol) else (got - want).abs() / tol)
                      .nan_to_num(0, 0, 0).max())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {worst:.2f} of the tolerance, "
                             f"first at {i}: {got.flatten()[i].item()} for {want.flatten()[i].item()}")


def tolerance(want, dtype, extra=0.0):
    scale = float(want[want.isfinite()].abs().max()) if want.isfinite().any() else 0.0
    return (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 1e-5 * scale + extra + 1e-30


# ---- norms and rotation -----------------------------------------------------------------------------

QK_CASES = [
    # T, Hq, Hk, D, rope, interleaved, dtype, layout
    (1, 32, 8, 128, 128, False, BF16, "contiguous"),
    (0, 4, 2, 64, 64, False, BF16, "contiguous"),
    (5, 4, 1, 64, 64, True, BF16, "padded"),
    (33, 5, 3, 128, 64, False, BF16, "padded"),
    (17, 3, 2, 256, 256, False, BF16, "contiguous"),
    (257, 7, 7, 80, 48, True, F32, "contiguous"),
    (64, 2, 2, 96, 96, False, F32, "padded"),
    (9, 6, 2, 24, 8, False, BF16, "contiguous"),
    (31, 3, 1, 128, 128, False, BF16, "odd"),
    (31, 3, 1, 128, 128, True, F32, "odd"),
    (6, 2, 2, 7, 4, False, BF16, "contiguous"),
    (6, 2, 2, 7, 6, True, F32, "contiguous"),
    (4, 1, 1, 1, 0, False, F32, "contiguous"),
    (11, 2, 0, 64, 64, False, BF16, "contiguous"),
    (3, 2, 1, 250, 250, True, BF16, "contiguous"),
    (2, 2, 1, 12, 12, False, BF16, "contiguous"),
    (2049, 9, 2, 128, 128, False, BF16, "contiguous"),
]


def qk_inputs(T, Hq, Hk, D, rope, dtype, layout, seed=0):
    g = gen(seed)
    q, k, gq, gk = (Guarded(T, h, D, dtype, layout).view for h in (Hq, Hk, Hq, Hk))
    for x in (q, k, gq, gk):
        x.copy_(randn(g, *x.shape))
    wq, wk = 1 + 0.3 * randn(g, D), 1 + 0.3 * randn(g, D)
    rows = T + 5
    cs = torch.cat([randn(g, rows, rope)], 1) if rope else None     # any numbers: a rotation is not assumed
    pos = torch.randint(0, rows, (T,), generator=g, device="cuda", dtype=torch.int32)
    return q, k, gq, gk, wq.to(dtype), wk.to(dtype), cs, pos


@pytest.mark.parametrize("T,Hq,Hk,D,rope,interleaved,dtype,layout", QK_CASES)
def test_qk_norm_rope_and_its_gradient(ctx, T, Hq, Hk, D, rope, interleaved, dtype, layout):
    q, k, gq, gk, wq, wk, cs, pos = qk_inputs(T, Hq, Hk, D, rope, dtype, layout)
    outs = [Guarded(T, h, D, dtype, layout) for h in (Hq, Hk, Hq, Hk)]
    yq, yk, dq, dk = (o.view for o in outs)
    kw = dict(eps=1e-5, interleaved=interleaved)
    ctx.slidedp_qk_norm_rope(q, k, wq, wk, cs, pos, yq, yk, **kw)
    dwq, dwk = (torch.full((D,), 9.0, device="cuda") for _ in range(2))
    ws = torch.empty(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8, device="cuda")
    ctx.slidedp_qk_norm_rope_backward(q, k, wq, wk, cs, pos, gq, gk, dq, dk, dwq, dwk, ws, **kw)
    torch.cuda.synchronize()
    for o, what in zip(outs, ("q_out", "k_out", "dq", "dk")):
        o.check(what)
    for x, w, gy, y, dx, dw, what in ((q, wq, gq, yq, dq, dwq, "q"), (k, wk, gk, yk, dk, dwk, "k")):
        want = ref.qk_forward(x, w, cs, pos, 1e-5, interleaved)
        assert_close("y of " + what, y, want, tolerance(want, dtype))
        wdx, wdw = ref.qk_backward(x, w, cs, pos, 1e-5, interleaved, gy)
        assert_close("dx of " + what, dx, wdx, tolerance(wdx, dtype))
        # FP32 sums of T * H terms of size about 1
        assert_close("dw of " + what, dw, wdw, 1e-5 * max(1.0, math.sqrt(T * max(x.shape[1], 1))) * 4)


def test_qk_in_place_null_weights_positions_and_out_of_table(ctx):
    T, H, D = 37, 3, 64
    q, k, gq, gk, _, _, cs, pos = qk_inputs(T, H, H, D, D, BF16, "contiguous", seed=5)
    want = ref.qk_forward(q, None, cs, torch.arange(T, device="cuda"), 1e-6, False)
    wdx, _ = ref.qk_backward(q, None, cs, torch.arange(T, device="cuda"), 1e-6, False, gq)
    kq, kk = q.clone(), k.clone()
    ctx.slidedp_qk_norm_rope_backward(q, k, None, None, cs, None, gq, gk, gq, gk, None, None, None)
    ctx.slidedp_qk_norm_rope(q, k, None, None, cs, None, q, k)
    assert_close("in place", q, want, tolerance(want, BF16))
    assert_close("gradient in place", gq, wdx, tolerance(wdx, BF16))
    pos[3], pos[9] = -1, cs.shape[0]
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    ctx.slidedp_qk_norm_rope(kq, kk, None, None, cs, pos, yq, yk)
    assert yq[3].isnan().all() and yk[9].isnan().all()
    rest = [i for i in range(T) if i not in (3, 9)]
    assert not yq[rest].isnan().any()


def test_qk_zero_rows_and_large_values(ctx):
    D = 128
    q = torch.zeros(4, 2, D, dtype=BF16, device="cuda")
    q[1] = 1e15
    q[2, 0, 5] = math.inf
    q[3] = torch.arange(D, device="cuda") * 1e-12
    w = torch.ones(D, dtype=BF16, device="cuda")
    y, y2 = torch.empty_like(q), torch.empty_like(q)
    ctx.slidedp_qk_norm_rope(q, q, w, w, None, None, y, y2, eps=1e-6)
    want = ref.qk_forward(q, w, None, None, 1e-6, False)
    for t in (0, 1, 3):
        assert_close(f"row {t}", y[t], want[t], tolerance(want[t], BF16))
    assert y[2, 0].isnan().any() and not y[2, 1].isnan().any()


def test_qk_is_reproducible_and_follows_its_stream(ctx):
    q, k, gq, gk, wq, wk, cs, pos = qk_inputs(1500, 8, 2, 128, 128, BF16, "contiguous", seed=7)
    ws = torch.empty(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8, device="cuda")
    def once(stream=None):
        o = [torch.empty_like(q), torch.empty_like(k), torch.empty(128, device="cuda"), torch.empty(128, device="cuda")]
        ctx.slidedp_qk_norm_rope_backward(q, k, wq, wk, cs, pos, gq, gk, *o, ws, stream=stream)
        return o
    a = once()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = once()
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- attention -----------------------------------------------------------------------------------------

def attn_case(ctx, T, Hq, Hk, D, cu=None, prefix=None, causal=True, softcap=0.0, bias=False, layout="contiguous",
              seed=0, scale=None, spread=1.0):
    g = gen(seed)
    ins = [Guarded(T, h, D, BF16, layout).view for h in (Hq, Hk, Hk, Hq)]
    for x in ins:
        x.copy_(randn(g, *x.shape, scale=spread))
    q, k, v, do = ins
    outs = [Guarded(T, h, D, BF16, layout) for h in (Hq, Hq, Hk, Hk)]
    out, dq, dk, dv = (o.view for o in outs)
    lse = torch.full((Hq, T), 5.0, device="cuda")
    tens = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    slopes = 2.0 ** -torch.arange(1, Hq + 1, device="cuda").float() if bias else None
    kw = dict(cu_docs=tens(cu), prefix=tens(prefix), slopes=slopes, causal=causal, scale=scale, softcap=softcap)
    ctx.slidedp_attention(q, k, v, out, lse, **kw)
    ws = torch.full((ctx.slidedp_attention_workspace(q, k),), 255, dtype=torch.uint8, device="cuda")
    ctx.slidedp_attention_backward(q, k, v, out, lse, do, dq, dk, dv, ws, **kw)
    torch.cuda.synchronize()
    for o, what in zip(outs, ("out", "dq", "dk", "dv")):
        o.check(what)
    ok = ref.visible(T, cu, prefix, causal, "cuda")
    want = ref.attention(q, k, v, D ** -0.5 if scale is None else scale, ok, softcap, slopes, do)
    assert_close("lse", lse, want["lse"], 2e-5 + 2e-6 * want["lse"].abs().nan_to_num(posinf=0))
    for n, got in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert_close(n, got, want[n], tolerance(want[n], BF16, want[n + "_bound"]))
    return dict(q=q, k=k, v=v, do=do, out=out, lse=lse, dq=dq, dk=dk, dv=dv, want=want, kw=kw)


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_lengths(ctx, T, D):
    attn_case(ctx, T, 4, 2, D, seed=T)


@pytest.mark.parametrize("D", [8, 16, 24, 40, 72, 80, 96, 104, 120])
def test_attention_head_dims(ctx, D):
    attn_case(ctx, 200, 2, 1, D, seed=D)


@pytest.mark.parametrize("D,layout", [(1, "contiguous"), (20, "contiguous"), (136, "contiguous"), (160, "padded"),
                                      (256, "contiguous"), (64, "odd"), (128, "odd"), (33, "odd")])
def test_attention_views_the_tensor_cores_do_not_take(ctx, D, layout):
    attn_case(ctx, 77, 4, 2, D, cu=[0, 10, 77], layout=layout, seed=D)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (8, 1), (5, 5), (12, 4), (40, 8)])
def test_attention_head_groups(ctx, Hq, Hk):
    attn_case(ctx, 150, Hq, Hk, 64, cu=[0, 70, 150], layout="padded", seed=Hq)


MASKS = [
    ([0, 300], None), ([0, 1, 2, 3, 300], None), ([0, 128, 256, 300], None), ([0, 0, 5, 5, 5, 299, 300, 300], None),
    ([0, 100, 250], None),                        # padding at the end
    ([40, 100, 250], None),                       # and at the start
    ([0], None), ([0, 0], None), ([300, 300], None),   # no token in any document: every row is empty
    ([0, 130, 300], [0, 300]), ([0, 130, 300], [130, 1]), ([0, 130, 290], [50, 100]), ([0, 300], [-4]),
    (list(range(0, 301, 3)), None), (list(range(301)), None),
]


@pytest.mark.parametrize("cu,prefix", MASKS)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_masks(ctx, cu, prefix, causal):
    attn_case(ctx, 300, 2, 1, 64, cu=cu, prefix=prefix, causal=causal, seed=len(cu))


@pytest.mark.parametrize("softcap,bias,causal,prefix", [
    (5.0, False, True, None), (30.0, True, True, [60, 20]), (0.0, True, False, None), (2.0, True, False, None),
    (0.0, True, True, [100, 10])])
@pytest.mark.parametrize("D", [64, 128, 96, 132])
def test_attention_cap_and_bias(ctx, softcap, bias, causal, prefix, D):
    attn_case(ctx, 280, 4, 2, D, cu=[0, 150, 270], prefix=prefix, causal=causal, softcap=softcap, bias=bias, seed=D,
              spread=1.5)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_longer_than_many_tiles(ctx, D):
    attn_case(ctx, 1531, 4, 1, D, cu=[0, 700, 1500], prefix=[300, 0], seed=2)


@pytest.mark.parametrize("D", [64, 128, 144])
def test_attention_large_and_small_scores(ctx, D):
    """Scores of several hundred (one key takes a row), equal scores, and a scale of zero or below."""
    attn_case(ctx, 190, 2, 1, D, scale=3.0, seed=11)
    attn_case(ctx, 190, 2, 1, D, scale=0.0, seed=12)
    attn_case(ctx, 190, 2, 1, D, scale=-0.2, seed=13)


def test_attention_rising_scores_rescale_every_tile(ctx):
    """Keys whose scores grow along the sequence: the running maximum moves in every tile."""
    T, D = 700, 64
    q = torch.full((T, 1, D), 1.0, dtype=BF16, device="cuda")
    k = (torch.arange(T, device="cuda") / 8.0)[:, None, None].expand(T, 1, D).to(BF16).contiguous()
    v = randn(gen(3), T, 1, D, dtype=BF16)
    out, lse = torch.empty_like(q), torch.empty(1, T, device="cuda")
    for sign in (1.0, -1.0):
        ctx.slidedp_attention(q * sign, k, v, out, lse)
        want = ref.attention(q * sign, k, v, D ** -0.5, ref.visible(T, None, None, True, "cuda"))
        assert_close("out", out, want["out"], tolerance(want["out"], BF16, want["out_bound"]))
        assert_close("lse", lse, want["lse"], 1e-3 + 2e-6 * want["lse"].abs())   # scores up to 700: 2^-24 of them


def test_attention_nan_stays_in_its_document(ctx):
    T, D = 260, 64
    g = gen(9)
    q, k, v = randn(g, T, 2, D, dtype=BF16), randn(g, T, 2, D, dtype=BF16), randn(g, T, 2, D, dtype=BF16)
    cu = torch.tensor([0, 130, 200], dtype=torch.int32, device="cuda")
    clean, lse0 = torch.empty_like(q), torch.empty(2, T, device="cuda")
    ctx.slidedp_attention(q, k, v, clean, lse0, cu_docs=cu)
    k2, v2 = k.clone(), v.clone()
    k2[140, 0], v2[140, 0] = math.nan, math.inf
    k2[230], v2[230] = math.nan, math.nan          # padding
    out, lse = torch.empty_like(q), torch.empty(2, T, device="cuda")
    ctx.slidedp_attention(q, k2, v2, out, lse, cu_docs=cu)
    assert out[140:200, 0].isnan().any(1).all()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[140:200] = False
    assert torch.equal(lse[:, keep], lse0[:, keep])
    assert torch.equal(lse[1], lse0[1])
    assert torch.all(out[200:] == 0) and torch.all(lse[:, 200:] == -math.inf)


def test_attention_is_reproducible_and_follows_its_stream(ctx):
    a = attn_case(ctx, 900, 8, 2, 128, cu=[0, 500, 900], seed=21)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = torch.empty_like(a["out"]), torch.empty_like(a["lse"])
        ctx.slidedp_attention(a["q"], a["k"], a["v"], out, lse, **a["kw"])
        dq, dk, dv = torch.empty_like(a["dq"]), torch.empty_like(a["dk"]), torch.empty_like(a["dv"])
        ws = torch.empty(ctx.slidedp_attention_workspace(a["q"], a["k"]), dtype=torch.uint8, device="cuda")
        ctx.slidedp_attention_backward(a["q"], a["k"], a["v"], out, lse, a["do"], dq, dk, dv, ws, **a["kw"])
    side.synchronize()
    for n, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(x, a[n]), n


def test_attention_offsets_outside_the_sequence_are_clamped(ctx):
    T, D = 150, 64
    g = gen(31)
    q, k, v = (randn(g, T, 1, D, dtype=BF16) for _ in range(3))
    a, b, la, lb = torch.empty_like(q), torch.empty_like(q), torch.empty(1, T, device="cuda"), torch.empty(1, T, device="cuda")
    ctx.slidedp_attention(q, k, v, a, la, cu_docs=torch.tensor([-50, 60, 9000], dtype=torch.int32, device="cuda"))
    ctx.slidedp_attention(q, k, v, b, lb, cu_docs=torch.tensor([0, 60, T], dtype=torch.int32, device="cuda"))
    assert torch.equal(a, b) and torch.equal(la, lb)


# ---- distillation ------------------------------------------------------------------------------------------

def distill_inputs(N, V, K, dtype, seed, stride=0, offset=0):
    g = gen(seed)
    whole = torch.full((N * (V + stride) + offset + 64,), 7.0, dtype=dtype, device="cuda")
    z = whole[offset:offset + N * (V + stride)].view(N, V + stride)[:, :V]
    z.copy_(randn(g, N, V, scale=3.0))
    ids = torch.randint(0, V, (N, K), generator=g, device="cuda", dtype=torch.int32)
    t = randn(g, N, K, scale=2.0)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    if K > 2:
        ids[0] = ids[0, 0]                # every entry the same
        ids[-1, 1] = ids[-1, 0]           # a repeat
        ids[N // 2, :2] = torch.tensor([-1, V], dtype=torch.int32)
        ids[N // 3] = -7                  # no entry at all
    labels[::3] = -100
    if N > 4:
        labels[4] = V
        if K:
            labels[1] = ids[1, 0]
    return z, ids, t, labels, torch.rand(N, generator=g, device="cuda") - 0.3


def distill_check(ctx, z, ids, t, labels, gr, tau, wt, wl, in_place=False, out_shift=0):
    N, V = z.shape
    dtype = z.dtype
    wloss, wlse, wdz = ref.distill(z.cpu(), ids.cpu(), t.cpu(), None if labels is None else labels.cpu(), tau, wt, wl,
                                   None if gr is None else gr.cpu())
    kw = dict(temperature=tau, w_teacher=wt, w_label=wl)
    zmax = float(z.float().abs().max()) if z.numel() else 0.0
    # FP32 logarithms of size zmax / tau + 12, weighted by tau^2
    ltol = 1e-6 * (1 + abs(wt) * tau * tau * (zmax / tau + 12) + abs(wl) * (zmax + 12)) * 4
    gmax = 1.0 if gr is None else float(gr.abs().max())
    # a probability is exp of an argument of that size: relative error 1e-6 times it; entries cancel against q
    gtol = (2.0 ** -8 * wdz.abs() if dtype == BF16 else 1e-5 * wdz.abs()) + 4e-6 * gmax * (abs(wt) * tau + abs(wl)) + 1e-30
    def buffers():
        whole = torch.full((N * V + out_shift + 64,), 7.0, dtype=dtype, device="cuda")
        return whole, whole[out_shift:out_shift + N * V].view(N, V)
    loss, lse = torch.full((N,), 9.0, device="cuda"), torch.full((2, N), 9.0, device="cuda")
    ctx.slidedp_distill_loss(z, ids, t, labels, loss, lse, **kw)
    assert_close("loss", loss, wloss, ltol)
    assert_close("lse", lse, wlse, 1e-6 * (zmax / tau + zmax + 12))
    whole, dz = buffers()
    ctx.slidedp_distill_loss_backward(z, ids, t, labels, lse, gr, dz, **kw)
    assert_close("backward", dz.cpu(), wdz, gtol)
    assert torch.all(whole[:out_shift] == 7.0) and torch.all(whole[out_shift + N * V:] == 7.0)
    whole, dz = buffers()
    if in_place:
        dz = z
    loss2, lse2 = torch.full((N,), 9.0, device="cuda"), torch.full((2, N), 9.0, device="cuda")
    ctx.slidedp_distill_step(z, ids, t, labels, gr, loss2, lse2, dz, **kw)
    assert_close("step loss", loss2, wloss, ltol)
    assert_close("step lse", lse2, wlse, 1e-6 * (zmax / tau + zmax + 12))
    assert_close("step gradient", dz.cpu(), wdz, gtol)
    assert torch.all(whole[:out_shift] == 7.0) and torch.all(whole[out_shift + N * V:] == 7.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (1, 2, 1), (5, 7, 3), (6, 1000, 8), (7, 8191, 20), (5, 16385, 512), (5, 33333, 0),
                                   (6, 131072, 64), (5, 100003, 100)])
def test_distill_sizes(ctx, dtype, N, V, K):
    distill_check(ctx, *distill_inputs(N, V, K, dtype, seed=V + K), tau=1.0, wt=1.0, wl=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau,wt,wl", [(1.0, 0.3, 0.7), (2.5, 0.6, 0.4), (0.5, 1.0, 1.0), (3.0, 0.0, 1.0), (1.0, 0.0, 1.0),
                                       (4.0, 1.0, 0.0)])
def test_distill_mixes(ctx, dtype, tau, wt, wl):
    distill_check(ctx, *distill_inputs(9, 5003, 16, dtype, seed=int(tau * 10)), tau=tau, wt=wt, wl=wl)


@pytest.mark.parametrize("dtype,stride,offset,shift", [(BF16, 1, 0, 0), (BF16, 3, 5, 1), (F32, 1, 1, 2), (BF16, 8, 8, 8), (F32, 0, 3, 3)])
def test_distill_any_alignment_and_stride(ctx, dtype, stride, offset, shift):
    distill_check(ctx, *distill_inputs(6, 4099, 9, dtype, seed=stride, stride=stride, offset=offset), tau=1.5, wt=0.5,
                  wl=0.5, out_shift=shift)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distill_in_place_without_labels_or_row_gradients(ctx, dtype):
    z, ids, t, labels, gr = distill_inputs(6, 70001, 12, dtype, seed=8)
    distill_check(ctx, z, ids, t, None, None, tau=2.0, wt=1.0, wl=0.5, in_place=True)


def test_distill_rows_longer_than_a_cluster_holds(ctx):
    """FP32 rows of 2 MB do not fit eight blocks' shared memory: the step reads them twice."""
    z, ids, t, labels, gr = distill_inputs(3, 500009, 5, F32, seed=18)
    distill_check(ctx, z, ids, t, labels, gr, tau=1.3, wt=0.5, wl=0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distill_masked_logits(ctx, dtype):
    """-inf and the type's lowest value in most places, far-off rows, and a teacher entry with no mass."""
    z, ids, t, labels, gr = distill_inputs(8, 3001, 6, dtype, seed=28)
    z[0, 100:] = -math.inf
    z[1, 50:] = torch.finfo(dtype).min
    z[2] -= 20000.0
    z[3] = torch.finfo(dtype).min
    ids[:, :] = torch.arange(6, device="cuda", dtype=torch.int32)
    labels[:] = 3
    t[4, 2] = -math.inf
    t[5, :] = -math.inf
    z[4, 2] = -math.inf
    z[6] = 0.0
    rows = torch.tensor([0, 1, 2, 4, 5, 6, 7])
    wloss, wlse, wdz = ref.distill(z[rows].cpu(), ids[rows].cpu(), t[rows].cpu(), labels[rows].cpu(), 2.0, 0.5, 0.5, gr[rows].cpu())
    loss, lse, dz = torch.empty(8, device="cuda"), torch.empty(2, 8, device="cuda"), torch.empty_like(z)
    ctx.slidedp_distill_step(z, ids, t, labels, gr, loss, lse, dz, temperature=2.0, w_teacher=0.5, w_label=0.5)
    assert_close("loss", loss[rows].cpu(), wloss, 1e-4 + 1e-6 * wloss.abs())
    # row 2's logits are near -2e4: an FP32 lse of that size is good to 2e-3
    assert_close("lse", lse[:, rows].cpu(), wlse, 1e-5 + 1e-6 * wlse.abs())
    assert_close("gradient", dz[rows].cpu(), wdz, 2.0 ** -8 * wdz.abs() + 1e-5)
    # a row of nothing but the lowest value is a uniform distribution
    assert abs(float(dz[3, 7]) / (float(gr[3]) * (0.5 * 2.0 + 0.5) / 3001) - 1) < 1e-2


def test_distill_nan_and_infinite_rows_stay_alone(ctx):
    z, ids, t, labels, gr = distill_inputs(4, 2000, 4, F32, seed=38)
    ids[:] = torch.arange(4, device="cuda", dtype=torch.int32)
    clean = torch.empty_like(z)
    loss, lse = torch.empty(4, device="cuda"), torch.empty(2, 4, device="cuda")
    ctx.slidedp_distill_step(z, ids, t, labels, gr, loss, lse, clean)
    z[1, 77] = math.nan
    z[2, 99] = math.inf
    dz, loss2 = torch.empty_like(z), torch.empty(4, device="cuda")
    ctx.slidedp_distill_step(z, ids, t, labels, gr, loss2, lse, dz)
    assert dz[1].isnan().all() and dz[2].isnan().any() and loss2[1].isnan() and loss2[2].isnan()
    assert torch.equal(dz[0], clean[0]) and torch.equal(dz[3], clean[3]) and torch.equal(loss2[3], loss[3])


def test_distill_gradient_matches_differences_of_the_loss(ctx):
    z, ids, t, labels, gr = distill_inputs(5, 300, 7, F32, seed=48)
    e = randn(gen(49), 5, 300)
    kw = dict(temperature=1.5, w_teacher=0.7, w_label=0.3)
    def f(y):
        loss, lse = torch.empty(5, device="cuda"), torch.empty(2, 5, device="cuda")
        ctx.slidedp_distill_loss(y, ids, t, labels, loss, lse, **kw)
        return loss.double()
    h = 2.0 ** -6
    num = (f(z + h * e) - f(z - h * e)) / (2 * h)
    loss, lse, dz = torch.empty(5, device="cuda"), torch.empty(2, 5, device="cuda"), torch.empty_like(z)
    ctx.slidedp_distill_step(z, ids, t, labels, None, loss, lse, dz, **kw)
    # FP32 losses near 20 over 2 h = 2^-5: 20 * 2^-23 * 32; and h^2 times a third derivative of order 1
    assert_close("directional derivative", (dz * e).sum(1), num, 5e-4)


# ---- refusals -----------------------------------------------------------------------------------------------

def test_refusals_leave_outputs_alone(ctx, sd):
    T, H, D = 4, 2, 64
    mk = lambda *s, dtype=BF16: torch.full(s, 3.0, dtype=dtype, device="cuda")  # noqa: E731
    q, k, y = mk(T, H, D), mk(T, H, D), mk(T, H, D)
    cs, pos = mk(4, D, dtype=F32), torch.zeros(T, dtype=torch.int32, device="cuda")
    w = mk(D)
    for bad in (dict(q=q.float()), dict(q=q[..., ::2]), dict(w_q=mk(D + 1)), dict(w_q=w.float()), dict(cos_sin=cs.double()),
                dict(positions=pos.long()), dict(positions=pos[:3]), dict(q_out=mk(T, H + 1, D)), dict(k=mk(T + 1, H, D))):
        args = dict(q=q, k=k, w_q=w, w_k=w, cos_sin=cs, positions=pos, q_out=y, k_out=y)
        with pytest.raises((TypeError, ValueError)):
            ctx.slidedp_qk_norm_rope(**{**args, **bad})
    for bad, status in ((dict(cos_sin=mk(4, D + 2, dtype=F32)), sd.ERR_INVALID_ARG), (dict(cos_sin=mk(4, 63, dtype=F32)), sd.ERR_INVALID_ARG),
                        (dict(cos_sin=mk(3, D, dtype=F32), positions=None), sd.ERR_INVALID_ARG), (dict(eps=-1.0), sd.ERR_INVALID_ARG)):
        args = dict(q=q, k=k, w_q=w, w_k=w, cos_sin=cs, positions=pos, q_out=y, k_out=y)
        with pytest.raises(sd.SlideDPError) as e:
            ctx.slidedp_qk_norm_rope(**{**args, **bad})
        assert e.value.status == status
    lse = mk(H, T, dtype=F32)
    for bad in (dict(lse=mk(T, H, dtype=F32)), dict(k=mk(T, H, D, dtype=F32)), dict(v=mk(T, 1, D)), dict(out=mk(T, H, 32)),
                dict(cu_docs=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(slopes=mk(H + 1, dtype=F32)),
                dict(cu_docs=torch.zeros(3, dtype=torch.int32, device="cuda"), prefix=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            ctx.slidedp_attention(**{**dict(q=q, k=k, v=k, out=y, lse=lse), **bad})
    for bad in (dict(scale=math.nan), dict(softcap=-2.0), dict(k=mk(T, 3, D), v=mk(T, 3, D)),
                dict(prefix=torch.zeros(1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(sd.SlideDPError):
            ctx.slidedp_attention(**{**dict(q=q, k=k, v=k, out=y, lse=lse), **bad})
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k) + 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        ctx.slidedp_attention_backward(q, k, k, y, lse, y, y, y, y, ws[:8])
    with pytest.raises(sd.SlideDPError) as e:
        ctx.slidedp_attention_backward(q, k, k, y, lse, y, y, y, y, ws[8:])
    assert e.value.status == sd.ERR_MISALIGNED
    z, ids, t = mk(3, 50), torch.zeros(3, 4, dtype=torch.int32, device="cuda"), mk(3, 4, dtype=F32)
    loss, l2 = mk(3, dtype=F32), mk(2, 3, dtype=F32)
    for bad in (dict(logits=z.half()), dict(teacher_ids=ids.long()), dict(teacher_logits=t.bfloat16()), dict(loss=mk(4, dtype=F32)),
                dict(lse=mk(3, 2, dtype=F32)), dict(labels=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(logits=z[:, ::2])):
        with pytest.raises((TypeError, ValueError)):
            ctx.slidedp_distill_loss(**{**dict(logits=z, teacher_ids=ids, teacher_logits=t, labels=None, loss=loss, lse=l2), **bad})
    for bad in (dict(temperature=0.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(w_teacher=math.nan), dict(w_label=math.inf),
                dict(teacher_ids=torch.zeros(3, 513, dtype=torch.int32, device="cuda"), teacher_logits=mk(3, 513, dtype=F32))):
        with pytest.raises(sd.SlideDPError):
            ctx.slidedp_distill_loss(**{**dict(logits=z, teacher_ids=ids, teacher_logits=t, labels=None, loss=loss, lse=l2), **bad})
    torch.cuda.synchronize()
    assert torch.all(y == 3.0) and torch.all(lse == 3.0) and torch.all(loss == 3.0) and torch.all(l2 == 3.0)


def test_sizes_of_zero_and_injected_failures(ctx, sd):
    none = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    i32 = torch.int32
    q = none(0, 4, 64)
    ctx.slidedp_attention(q, q, q, q, none(4, 0, dtype=F32))
    ctx.slidedp_attention_backward(q, q, q, q, none(4, 0, dtype=F32), q, q, q, q, none(64, dtype=torch.uint8))
    ctx.slidedp_distill_step(none(0, 9), none(0, 2, dtype=i32), none(0, 2, dtype=F32), None, None, none(0, dtype=F32),
                             none(2, 0, dtype=F32), none(0, 9))
    # every guarded call in turn: reported, nothing of it queued, and the context usable afterwards
    g = gen(77)
    q, k = randn(g, 40, 4, 64, dtype=BF16), randn(g, 40, 2, 64, dtype=BF16)
    out, lse, ws = torch.empty_like(q), none(4, 40, dtype=F32), none(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    dw = [none(64, dtype=F32) for _ in range(2)]
    ws2 = none(ctx.slidedp_qk_norm_rope_workspace(q, k), dtype=torch.uint8)
    z, ids, t = randn(g, 3, 500), torch.zeros(3, 2, dtype=i32, device="cuda"), randn(g, 3, 2)
    loss, l2, dz = none(3, dtype=F32), none(2, 3, dtype=F32), torch.empty_like(z)
    calls = [lambda: ctx.slidedp_attention(q, k, k, out, lse),
             lambda: ctx.slidedp_attention_backward(q, k, k, out, lse, q, dq, dk, dv, ws),
             lambda: ctx.slidedp_qk_norm_rope(q, k, None, None, None, None, dq, dk),
             lambda: ctx.slidedp_qk_norm_rope_backward(q, k, None, None, None, None, q, k, dq, dk, *dw, ws2),
             lambda: ctx.slidedp_distill_loss(z, ids, t, None, loss, l2),
             lambda: ctx.slidedp_distill_loss_backward(z, ids, t, None, l2, None, dz),
             lambda: ctx.slidedp_distill_step(z, ids, t, None, None, loss, l2, dz)]
    for call in calls:
        for nth in range(1, 20):
            ctx.slidedp_test_fail_nth_call(nth)
            try:
                call()
            except sd.SlideDPError as e:
                assert e.status == sd.ERR_CUDA
                continue
            finally:
                ctx.slidedp_test_fail_nth_call(0)
            break
        else:
            raise AssertionError("more than 19 guarded calls")
        assert nth > 1
        call()
    torch.cuda.synchronize()
    attn_case(ctx, 60, 4, 2, 64, seed=1)
