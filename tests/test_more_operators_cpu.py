"""Embedding, block norms, policy loss and clipping without a GPU: argument checks through the C ABI, and the 64-bit formulas that the
GPU tests compare with, themselves checked against differences."""
import ctypes
import math

import pytest
import torch

import more_operators_ref as ref

F64 = torch.float64


@pytest.fixture(scope="module")
def sd():
    import paper_2609_34162_b200.slidedp as sd
    return sd


def difference(f, x, direction, h=1e-5):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_embedding_formula_matches_differences():
    g = torch.Generator().manual_seed(1)
    ids = torch.tensor([2, 0, 2, -1, 5, 4, 2], dtype=torch.int32)
    table, e = (torch.randn(5, 3, generator=g, dtype=F64) for _ in range(2))
    dy = torch.randn(7, 3, generator=g, dtype=F64)
    f = lambda t: (ref.embedding(t, ids, 1.7) * dy).sum()  # noqa: E731
    d, size, count = ref.embedding_backward(ids, dy, 5, 1.7)
    assert abs(difference(f, table, e) - (d * e).sum()) < 1e-7
    assert count.flatten().tolist() == [1, 0, 3, 0, 1] and torch.all(size >= d.abs())


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate,sigmoid", [(None, False), (1, False), (1, True), (2, False), (2, True)])
def test_block_norm_formula_matches_differences(post, gate, sigmoid):
    g = torch.Generator().manual_seed(7)
    T, H = 4, 6
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=F64)  # noqa: E731
    a = dict(x=rnd(T, H), y=rnd(T, H), w_post=rnd(H) if post else None, gate=None if gate is None else rnd(H) if gate == 1 else rnd(T, H),
             w_pre=rnd(H))
    gx, gh = rnd(T, H), rnd(T, H)

    def f(**kw):
        r = ref.block_norm(*{**a, **kw}.values(), 0.6, 1e-3, post, sigmoid)
        return (r["x_out"] * gx + r["h"] * gh).sum()

    r = ref.block_norm(*a.values(), 0.6, 1e-3, post, sigmoid, gx, gh, backward=True)
    for name, x in a.items():
        if x is None:
            continue
        e = rnd(*x.shape)
        d = r["d" + name]
        assert abs(difference(lambda t: f(**{name: t}), x, e) - (d * e).sum()) < 1e-7, name
        assert torch.all(r["d" + name + "_size"] >= d.abs() - 1e-12)


@pytest.mark.parametrize("tau,kl,with_old", [(1.0, 0.0, True), (0.7, 0.3, True), (1.3, 0.2, False)])
def test_policy_formula_matches_differences(tau, kl, with_old):
    g = torch.Generator().manual_seed(5)
    N, V = 40, 9
    z, e = (torch.randn(N, V, generator=g, dtype=F64) for _ in range(2))
    labels = torch.randint(-1, V + 1, (N,), generator=g)
    lp = torch.log_softmax(z / tau, 1).gather(1, labels.clamp(0, V - 1)[:, None])[:, 0]
    # ratios away from the edges 0.8 and 1.3, so that differences do not cross them
    old = lp - torch.tensor([-0.5, -0.1, 0.0, 0.1, 0.5])[torch.arange(N) % 5] if with_old else None
    adv, refp, gr = torch.randn(N, generator=g, dtype=F64), lp + 0.3 * torch.randn(N, generator=g, dtype=F64), torch.rand(N, generator=g, dtype=F64)
    if not with_old:      # the ratio is 1 with logp's own gradient: the loss's value does not move with it
        olds = lp
        f = lambda t: (ref.policy(t, labels, olds, refp, adv, tau, 0.2, 0.3, kl)[0][0] * gr).sum()  # noqa: E731
    else:
        f = lambda t: (ref.policy(t, labels, old, refp, adv, tau, 0.2, 0.3, kl)[0][0] * gr).sum()  # noqa: E731
    (_, _, dz), _ = ref.policy(z, labels, old, refp, adv, tau, 0.2, 0.3, kl, gr)
    assert abs(difference(f, z, e) - (dz * e).sum()) < 1e-6
    assert not dz[(labels < 0) | (labels >= V)].any()


def test_clip_formula():
    out, res = ref.clip([torch.tensor([3.0]), torch.tensor([0.0, -4.0])], 2.0, 5.0)
    assert res[:2] == [100.0, 10.0] and abs(res[2] - 0.5) < 1e-6 and res[3] == 0.0
    assert abs(float(out[1][1]) + 4.0) < 1e-6
    assert ref.clip([torch.tensor([1.0])], 1.0, 0.0)[1] == [1.0, 1.0, 1.0, 0.0]


def test_workspaces_and_refused_arguments(sd):
    lib = sd._lib
    ok = dict(tokens=70, vocab=100, hidden=64, dtype=0, grad_dtype=1, accumulate=0, scale=1.0)
    em = lambda **kw: lib.slidedp_embedding_workspace(ctypes.byref(sd._EmbeddingArgs(**{**ok, **kw})))  # noqa: E731
    assert em() > 0 and em(tokens=0) > 0 and em(hidden=1, vocab=1) > 0 and em(tokens=1 << 30, vocab=1 << 30) > 1 << 34
    for bad in (dict(tokens=-1), dict(vocab=0), dict(hidden=0), dict(dtype=2), dict(grad_dtype=-1), dict(accumulate=2), dict(scale=math.nan),
                dict(scale=1e39), dict(tokens=(1 << 30) + 1), dict(vocab=(1 << 30) + 1), dict(hidden=(1 << 20) + 1)):
        assert em(**bad) == 0, bad
    ok = dict(tokens=5, hidden=64, dtype=0, has_y=1, post_norm=1, pre_norm=1, gate_kind=0, gate_sigmoid=0, residual_scale=1.0, eps=1e-6)
    bn = lambda **kw: lib.slidedp_block_norm_workspace(ctypes.byref(sd._BlockNormArgs(**{**ok, **kw})))  # noqa: E731
    assert bn() > 0 and bn(hidden=16384) > 0 and bn(has_y=0, post_norm=0) > 0 and bn(gate_kind=2, gate_sigmoid=1) > 0 and bn(eps=0.0) > 0
    for bad in (dict(tokens=-1), dict(hidden=0), dict(hidden=16385), dict(dtype=2), dict(has_y=2), dict(has_y=0), dict(post_norm=-1), dict(pre_norm=2),
                dict(gate_kind=3), dict(gate_sigmoid=1), dict(residual_scale=math.inf), dict(eps=-1.0), dict(eps=math.nan), dict(eps=1e-50),
                dict(has_y=0, post_norm=0, pre_norm=0), dict(has_y=0, post_norm=0, gate_kind=1)):
        assert bn(**bad) == 0, bad
    tensors = lambda *t: ((sd._Tensor * len(t))(*[sd._Tensor(*x, 0) for x in t]), len(t))  # noqa: E731
    cw = lambda *t: lib.slidedp_clip_grad_norm_workspace(*tensors(*t))  # noqa: E731
    assert cw((16, 5, 1), (18, 3, 0)) > 0 and cw((0, 0, 0)) > 0 and lib.slidedp_clip_grad_norm_workspace(None, 0) > 0
    for bad in ((16, -1, 0), (0, 1, 0), (17, 1, 0), (18, 1, 1), (16, 1, 2), (16, 1 << 45, 0)):
        assert cw(bad) == 0, bad
    assert lib.slidedp_clip_grad_norm_workspace(None, 1) == 0 and lib.slidedp_clip_grad_norm_workspace(None, -1) == 0
    # without a context nothing is looked at further
    assert lib.slidedp_embedding(None, None, *[None] * 4) == sd.ERR_INVALID_ARG
    assert lib.slidedp_embedding_backward(None, None, *[None] * 5) == sd.ERR_INVALID_ARG
    assert lib.slidedp_block_norm(None, None, *[None] * 8) == sd.ERR_INVALID_ARG
    assert lib.slidedp_block_norm_backward(None, None, *[None] * 14) == sd.ERR_INVALID_ARG
    assert lib.slidedp_policy_loss(None, None, *[None] * 8) == sd.ERR_INVALID_ARG
    assert lib.slidedp_policy_loss_backward(None, None, *[None] * 9) == sd.ERR_INVALID_ARG
    assert lib.slidedp_policy_step(None, None, *[None] * 10) == sd.ERR_INVALID_ARG
    assert lib.slidedp_clip_grad_norm(None, None, None, 0, 1.0, 1.0, None, None, None) == sd.ERR_INVALID_ARG


def test_the_header_is_c(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "use.c"
    src.write_text('#include "slidedp_ops.h"\n'
                   "int main(void) {\n"
                   "  slidedp_rows r = {0, 0};\n"
                   "  slidedp_tensor t = {0, 0, SLIDEDP_F32, 0};\n"
                   "  slidedp_embedding_args e = {4, 8, 16, SLIDEDP_BF16, SLIDEDP_F32, 0, 0, 1.0};\n"
                   "  slidedp_block_norm_args b = {4, 8, SLIDEDP_BF16, 1, 1, 1, 0, 0, 1.0, 1e-6};\n"
                   "  slidedp_policy_args p = {4, 8, SLIDEDP_BF16, 0, 8, 8, 1.0, 0.2, 0.2, 0.0};\n"
                   "  return slidedp_embedding(0, &e, &r, 0, &r, 0) != SLIDEDP_ERR_INVALID_ARG || slidedp_embedding_workspace(&e) == 0 ||\n"
                   "         slidedp_block_norm(0, &b, &r, &r, 0, 0, 0, &r, &r, 0) != SLIDEDP_ERR_INVALID_ARG ||\n"
                   "         slidedp_block_norm_workspace(&b) == 0 || slidedp_clip_grad_norm_workspace(&t, 1) == 0 ||\n"
                   "         slidedp_policy_loss(0, &p, 0, 0, 0, 0, 0, 0, 0, 0) != SLIDEDP_ERR_INVALID_ARG;\n}\n")
    pkg = os.path.join(root, "paper_2609_34162_b200")
    exe = tmp_path / "use"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe),
                    "-L", pkg, "-lslidedp", f"-Wl,-rpath,{pkg}"], check=True)
    subprocess.run([str(exe)], check=True)
