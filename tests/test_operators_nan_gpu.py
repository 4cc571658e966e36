"""NaN and infinities in what a row of attention sees and in what it does not see: the first must show, the second must not,
and neither may cost more than a multiple of an ordinary pass."""
import math
import random

import pytest
import torch

import operators_ref as ref
from test_operators_gpu import BF16, F32, assert_close, ctx, gen, randn, sd, tolerance  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs(T, Hq, Hk, D, seed):
    g = gen(seed)
    return [randn(g, T, h, D, dtype=BF16) for h in (Hq, Hk, Hk, Hq)]


def forward(ctx, q, k, v, **kw):
    out, lse = torch.empty_like(q), torch.empty(q.shape[1], q.shape[0], device="cuda")
    ctx.slidedp_attention(q, k, v, out, lse, **kw)
    return out, lse


MODES = [dict(), dict(slopes=True), dict(softcap=20.0), dict(softcap=0.5, slopes=True)]


def keywords(mode, heads):
    kw = dict(mode)
    if kw.get("slopes"):
        kw["slopes"] = 2.0 ** -torch.arange(1, heads + 1, device="cuda").float()
    return kw


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("mode", MODES, ids=["plain", "bias", "cap", "cap_bias"])
def test_a_nan_key_shows_in_every_row_that_sees_it(ctx, D, mode):
    T, Hq, Hk = 300, 4, 2
    q, k, v, _ = inputs(T, Hq, Hk, D, seed=D)
    kw = keywords(mode, Hq)
    want = ref.attention(q, k, v, D ** -0.5, ref.visible(T, None, None, True, "cuda"), kw.get("softcap", 0.0), kw.get("slopes"))
    for j in [*range(18), 127, 128, 130, 133, 143, 257, 299]:
        for value, also_v in ((math.nan, False), (math.nan, True)):
            k2, v2 = k.clone(), v.clone()
            k2[j, 1, 3] = value
            if also_v:
                v2[j, 1] = value
            out, lse = forward(ctx, q, k2, v2, **kw)
            assert out[j:, 2:].isnan().all() and lse[2:, j:].isnan().all(), j
            tol = tolerance(want["out"], BF16, want["out_bound"])
            assert_close("rows before it", out[:j], want["out"][:j], tol[:j])
            assert_close("the other heads", out[:, :2], want["out"][:, :2], tol[:, :2])
            rest = lse.clone()
            rest[2:, j:] = want["lse"][2:, j:].float()
            assert_close("lse", rest, want["lse"], 2e-5 + 2e-6 * want["lse"].abs())


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("mode", MODES, ids=["plain", "bias", "cap", "cap_bias"])
def test_a_nan_query_is_nan_whatever_it_sees(ctx, D, mode):
    T, H = 270, 2
    q, k, v, _ = inputs(T, H, H, D, seed=D + 1)
    for i in [0, 1, 2, 5, 131, 269]:
        q2 = q.clone()
        q2[i, 1] = math.nan
        out, lse = forward(ctx, q2, k, v, **keywords(mode, H))
        assert out[i, 1].isnan().all() and lse[1, i].isnan(), i
        assert int(out.isnan().any(-1).sum()) == 1 and int(lse.isnan().sum()) == 1, i


@pytest.mark.parametrize("D", [64, 128, 20])
def test_a_key_with_a_score_of_minus_infinity_weighs_nothing(ctx, D):
    """As if it were not there, wherever it lies; a row with nothing else is 0 / 0."""
    T, H = 200, 2
    q, k, v, _ = inputs(T, H, H, D, seed=D + 2)
    q[:, :, 0] = 1.0
    seen = ref.visible(T, None, None, True, "cuda")
    for js in ([0], [0, 1, 2], [5], [128], [199], [0, 127, 128, 150]):
        k2, ok = k.clone(), seen.clone()
        k2[js, :, 0] = -math.inf
        ok[:, js] = False
        want = ref.attention(q, k, v, D ** -0.5, ok)
        out, lse = forward(ctx, q, k2, v)
        some = ok.any(1)
        assert_close("out", out[some], want["out"][some], tolerance(want["out"], BF16, want["out_bound"])[some])
        assert out[~some].isnan().all() and torch.all(lse[:, ~some] == -math.inf)
        assert_close("lse", lse[:, some], want["lse"][:, some], 2e-5 + 2e-6 * want["lse"][:, some].abs())


def backward(ctx, q, k, v, out, lse, do, **kw):
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
    ctx.slidedp_attention_backward(q, k, v, out, lse, do, dq, dk, dv, ws, **kw)
    return dict(dq=dq, dk=dk, dv=dv)


def timed(f):
    best = math.inf
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        r = f()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return r, best


@pytest.mark.parametrize("Hq,Hk,D", [(8, 2, 128), (8, 2, 64), (3, 3, 96)])
@pytest.mark.parametrize("where", ["k", "v", "q", "do", "token"])
def test_one_nan_in_a_long_document(ctx, Hq, Hk, D, where):
    """At token t, in the first document of two: what it must and must not reach, and what it may cost."""
    T, cu, t, G, c = 2600, [0, 2500, 2600], 40, Hq // Hk, 3
    q, k, v, do = inputs(T, Hq, Hk, D, seed=7)
    kw = dict(cu_docs=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    want = ref.attention(q, k, v, D ** -0.5, ref.visible(T, cu, None, True, "cuda"), 0.0, None, do)
    (out, lse), clean_f = timed(lambda: forward(ctx, q, k, v, **kw))
    grads, clean_b = timed(lambda: backward(ctx, q, k, v, out, lse, do, **kw))
    for n, x in (("k", k), ("v", v), ("q", q), ("do", do)):
        if where == n:
            x[t, 0, c] = math.nan            # head 0, and as a key head the queries' heads 0 .. G - 1
        elif where == "token":
            x[t] = math.nan
    (out, lse), nan_f = timed(lambda: forward(ctx, q, k, v, **kw))
    got, nan_b = timed(lambda: backward(ctx, q, k, v, out, lse, do, **kw))
    ctx.slidedp_qk_norm_rope(q, k, None, None, None, None, q.clone(), k.clone())     # would tell of a wait that ran out
    got["out"] = out
    nans = {n: torch.zeros_like(x, dtype=torch.bool) for n, x in got.items()}
    doc, late, early = slice(0, 2500), slice(t, 2500), slice(0, t + 1)
    if where == "k":         # every later query's scores
        nans["out"][late, :G] = nans["dq"][late, :G] = nans["dk"][doc, 0] = nans["dv"][doc, 0] = True
    elif where == "v":       # one column of the outputs, and with it delta
        nans["out"][late, :G, c] = nans["dq"][late, :G] = nans["dk"][doc, 0] = True
    elif where == "q":       # one row
        nans["out"][t, 0] = nans["dq"][t, 0] = nans["dk"][early, 0] = nans["dv"][early, 0] = True
    elif where == "do":
        nans["dq"][t, 0] = nans["dk"][early, 0] = nans["dv"][early, 0, c] = True
    else:
        nans["out"][late] = nans["dq"][late] = nans["dk"][doc] = nans["dv"][doc] = True
    assert torch.equal(lse.isnan(), nans["out"].all(-1).T)
    for n, x in got.items():
        assert torch.equal(x.isnan(), nans[n]), n
        tol = tolerance(want[n], BF16, want[n + "_bound"])
        keep = ~nans[n]
        assert_close(n, x[keep], want[n][keep], tol[keep])
    # rows whose NaN is their own are left as they are; redoing them cost over a thousand times an ordinary pass
    assert nan_f < 10 * clean_f + 1.0
    assert nan_b < (10 if where in ("k", "v", "token") else 1000) * clean_b + 1.0


def apart(x):
    """The same values one element off alignment, where one warp walks the pairs that it sees and nothing else."""
    y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
    return y.copy_(x)


@pytest.mark.parametrize("seed", range(80))
def test_nan_and_infinities_are_where_the_visible_pairs_put_them(ctx, seed):
    """Random documents with NaN and infinities strewn in: which results are NaN, infinite or finite, as in the general kernels,
    and the finite ones as the definition has them without the strewn values (no row that is finite sees any)."""
    r = random.Random(seed)
    T, Hk, G, D = r.choice([1, 5, 130, 257, 300, 500, 700]), r.choice([1, 2, 3]), r.choice([1, 2, 4]), r.choice([8, 40, 64, 96, 128])
    docs = r.randint(0, 6)
    cu = sorted(r.randint(0, T) for _ in range(docs + 1)) if r.random() < 0.8 else None
    prefix = [r.randint(-2, T // 2) for _ in range(docs)] if cu is not None and docs and r.random() < 0.4 else None
    tens = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kw = dict(causal=r.random() < 0.7, softcap=r.choice([0.0, 0.0, 5.0]), scale=r.choice([None, None, 0.3, -0.1]), cu_docs=tens(cu),
              prefix=tens(prefix))
    if r.random() < 0.3:
        kw["slopes"] = 2.0 ** -torch.arange(1, Hk * G + 1, device="cuda").float()
    clean = inputs(T, Hk * G, Hk, D, seed)
    ins = [x.clone() for x in clean]
    for _ in range(r.choice([1, 1, 2, 6])):
        x, value, t, part = r.choice(ins), r.choice([math.nan, math.nan, math.inf, -math.inf]), r.randrange(T), r.random()
        h = r.randrange(x.shape[1])
        if part < 0.5:
            x[t, h, r.randrange(D)] = value
        elif part < 0.8:
            x[t, h] = value
        else:
            x[t] = value

    def both(ins, place):
        q, k, v, do = map(place, ins)
        out, lse = place(torch.zeros_like(q)), torch.empty(q.shape[1], T, device="cuda")
        res = dict(out=out, dq=place(torch.zeros_like(q)), dk=place(torch.zeros_like(k)), dv=place(torch.zeros_like(v)))
        ws = torch.empty(ctx.slidedp_attention_workspace(q, k), dtype=torch.uint8, device="cuda")
        ctx.slidedp_attention(q, k, v, out, lse, **kw)
        ctx.slidedp_attention_backward(q, k, v, out, lse, do, res["dq"], res["dk"], res["dv"], ws, **kw)
        return {**res, "lse": lse.T}
    got, general = both(ins, lambda x: x), both(ins, apart)
    scale = D ** -0.5 if kw["scale"] is None else kw["scale"]
    want = ref.attention(*clean[:3], scale, ref.visible(T, cu, prefix, kw["causal"], "cuda"), kw["softcap"], kw.get("slopes"), clean[3])
    for n, x in got.items():
        y = general[n]
        assert torch.equal(x.isnan(), y.isnan()), f"{n}: NaN"
        assert torch.equal(x.isinf(), y.isinf()) and torch.equal(x[x.isinf()], y[x.isinf()]), f"{n}: infinities"
        if n != "lse":
            tol = tolerance(want[n], BF16, want[n + "_bound"])
            # a score of -inf takes its key out of a row, a score gradient of a row that is NaN its query out of a sum: only rows
            # and keys of heads without any strewn value are as in the clean definition
            if not any((~a.isfinite()).any() for a in ins[:3]):
                keep = x.isfinite()
                assert_close(n, x[keep], want[n][keep], tol[keep])
