"""The fine-tuning operators without a GPU: argument checks through the C ABI, the mask's definition,
and the 64-bit formulas that the GPU tests compare with, themselves checked against differences."""
import ctypes
import math

import pytest
import torch

import operators_ref as ref


@pytest.fixture(scope="module")
def sd():
    import paper_2609_34162_b200.slidedp as sd
    return sd


def difference(f, x, direction, h=1e-5):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rope", [(8, 8), (10, 4), (7, 6), (5, 0)])
def test_norm_rotation_formula_matches_differences(D, rope, interleaved):
    g = torch.Generator().manual_seed(D * 10 + rope)
    x = torch.randn(3, 2, D, generator=g, dtype=torch.float64)
    w, dy, e = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((D,), x.shape, x.shape))
    cs = torch.randn(5, rope, generator=g, dtype=torch.float64) if rope else None
    pos = torch.tensor([4, 0, 2])
    f = lambda x_, w_: (ref.qk_forward(x_, w_, cs, pos, 1e-3, interleaved) * dy).sum()  # noqa: E731
    dx, dw = ref.qk_backward(x, w, cs, pos, 1e-3, interleaved, dy)
    # central differences of a smooth function of size O(10): h^2 f''' + 1e-16 f / h, far below 1e-7
    assert abs(difference(lambda y: f(y, w), x, e) - (dx * e).sum()) < 1e-7
    ew = torch.randn(D, generator=g, dtype=torch.float64)
    assert abs(difference(lambda y: f(x, y), w, ew) - (dw * ew).sum()) < 1e-7


@pytest.mark.parametrize("softcap,bias", [(0.0, False), (2.0, False), (0.0, True), (3.0, True)])
def test_attention_formula_matches_differences(softcap, bias):
    g = torch.Generator().manual_seed(3)
    T, Hq, Hk, D = 9, 4, 2, 5
    q, k, v, do = (torch.randn(T, h, D, generator=g, dtype=torch.float64) for h in (Hq, Hk, Hk, Hq))
    ok = ref.visible(T, [0, 4, 4, 8], [2, 0, 1], True)
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0]) if bias else None
    f = lambda a, b, c: (ref.attention(a, b, c, 0.7, ok, softcap, slopes)["out"] * do).sum()  # noqa: E731
    r = ref.attention(q, k, v, 0.7, ok, softcap, slopes, do)
    for n, x, args in (("dq", q, lambda y: (y, k, v)), ("dk", k, lambda y: (q, y, v)), ("dv", v, lambda y: (q, k, y))):
        e = torch.randn(x.shape, generator=g, dtype=torch.float64)
        assert abs(difference(lambda y: f(*args(y)), x, e) - (r[n] * e).sum()) < 1e-7
    assert torch.all(r["out"][8] == 0) and torch.all(r["lse"][:, 8] == -math.inf) and torch.all(r["dq"][8] == 0)


def test_distillation_formula_matches_differences():
    g = torch.Generator().manual_seed(4)
    N, V = 4, 11
    z, e = (torch.randn(N, V, generator=g, dtype=torch.float64) for _ in range(2))
    ids = torch.tensor([[1, 5, 1], [10, -1, 3], [-1, 11, -5], [2, 2, 2]])
    t = torch.randn(N, 3, generator=g, dtype=torch.float64)
    labels, gr = torch.tensor([3, -100, 2, 2]), torch.rand(N, generator=g, dtype=torch.float64)
    f = lambda y: (ref.distill(y, ids, t, labels, 1.7, 0.6, 0.4)[0] * gr).sum()  # noqa: E731
    dz = ref.distill(z, ids, t, labels, 1.7, 0.6, 0.4, gr)[2]
    assert abs(difference(f, z, e) - (dz * e).sum()) < 1e-7


def test_workspaces_and_refused_arguments(sd):
    lib = sd._lib
    ok = dict(tokens=5, heads_q=4, heads_k=2, head_dim=64, rope_dim=64, interleaved=0, dtype=0, table_rows=9, eps=1e-6)
    qk = lambda **kw: lib.slidedp_qk_norm_rope_workspace(ctypes.byref(sd._QkArgs(**{**ok, **kw})))  # noqa: E731
    assert qk() > 0 and qk(head_dim=1, rope_dim=0) > 0 and qk(heads_k=0) > 0
    for bad in (dict(tokens=-1), dict(head_dim=0), dict(head_dim=257), dict(rope_dim=63), dict(rope_dim=66),
                dict(rope_dim=-2), dict(heads_q=-1), dict(interleaved=2), dict(dtype=2), dict(dtype=-1),
                dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(table_rows=-1)):
        assert qk(**bad) == 0, bad
    ok = dict(tokens=5, heads_q=4, heads_kv=2, head_dim=64, causal=1, docs=1, scale=1.0, softcap=0.0)
    at = lambda **kw: lib.slidedp_attention_workspace(ctypes.byref(sd._AttnArgs(**{**ok, **kw})))  # noqa: E731
    assert at() == 4 * 128 * 8 and at(tokens=129) == 4 * 256 * 8
    for bad in (dict(tokens=-1), dict(heads_q=3), dict(heads_q=0), dict(heads_kv=0), dict(head_dim=0), dict(head_dim=257),
                dict(causal=2), dict(docs=2), dict(docs=0), dict(scale=math.nan), dict(scale=math.inf),
                dict(softcap=-1.0), dict(softcap=math.nan), dict(prefix=16), dict(cu_docs=17, docs=3)):
        assert at(**bad) == 0, bad
    # without a context nothing is looked at further
    assert lib.slidedp_qk_norm_rope(None, None, *[None] * 9) == sd.ERR_INVALID_ARG
    assert lib.slidedp_attention(None, None, *[None] * 6) == sd.ERR_INVALID_ARG
    assert lib.slidedp_attention_backward(None, None, *[None] * 11) == sd.ERR_INVALID_ARG
    assert lib.slidedp_distill_loss(None, None, *[None] * 7) == sd.ERR_INVALID_ARG
    assert lib.slidedp_distill_loss_backward(None, None, *[None] * 8) == sd.ERR_INVALID_ARG
    assert lib.slidedp_distill_step(None, None, *[None] * 9) == sd.ERR_INVALID_ARG


def test_factors_that_fp32_does_not_hold_are_refused(sd):
    """They would otherwise be used as zero (a cap that is silently off) or infinity."""
    lib = sd._lib
    ok = dict(tokens=5, heads_q=4, heads_kv=2, head_dim=64, causal=1, docs=1, scale=1.0, softcap=0.0)
    at = lambda **kw: lib.slidedp_attention_workspace(ctypes.byref(sd._AttnArgs(**{**ok, **kw})))  # noqa: E731
    for good in (dict(scale=1e30), dict(scale=-1e-30), dict(softcap=1e-20), dict(softcap=1e30), dict(scale=1e-300)):
        assert at(**good) > 0, good
    for bad in (dict(scale=1e39), dict(scale=-3.3e38), dict(softcap=1e-46), dict(softcap=1e39), dict(softcap=1e300), dict(scale=1e20, softcap=1e-20)):
        assert at(**bad) == 0, bad
    ok = dict(tokens=5, heads_q=4, heads_k=2, head_dim=64, rope_dim=64, interleaved=0, dtype=0, table_rows=9, eps=1e-6)
    qk = lambda **kw: lib.slidedp_qk_norm_rope_workspace(ctypes.byref(sd._QkArgs(**{**ok, **kw})))  # noqa: E731
    assert qk(eps=0.0) > 0 and qk(eps=1e-40) > 0 and qk(eps=1e39) == 0 and qk(eps=1e-50) == 0


def test_the_paper_path_does_without_the_operators_module():
    """Without _marshal (not built, or built for another torch) the binding imports; the operators say what is missing."""
    import os
    import subprocess
    import sys
    code = (
        "import sys\n"
        "class Block:\n"
        "    def find_spec(self, name, path=None, target=None):\n"
        "        if '_marshal' in name: raise ImportError('blocked ' + name)\n"
        "sys.meta_path.insert(0, Block())\n"
        "import paper_2609_34162_b200.slidedp as sd, torch\n"
        "assert sd.slidedp_state_bytes(1) == 16 and sd._marshal is None\n"
        "c = sd.Context.__new__(sd.Context); c._h = sd._vp(); c.device = 0\n"
        "x = torch.zeros(1, 1, 8)\n"
        "try: c.slidedp_qk_norm_rope(x, x, None, None, None, None, x, x)\n"
        "except ImportError as e: assert 'paper_2609_34162_b200.build' in str(e) and 'blocked' in str(e.__cause__)\n"
        "else: raise SystemExit('no ImportError')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_operators_module_is_of_this_torch(sd):
    import re
    assert sd._marshal.__name__.endswith("._marshal_torch_" + re.sub(r"\W", "_", torch.__version__))


def test_the_headers_are_c(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "use.c"
    src.write_text('#include "slidedp_ops.h"\n'
                   "int main(void) {\n"
                   "  slidedp_heads h = {0, 0, 0};\n"
                   "  slidedp_qk_args q = {0, 1, 1, 8, 0, 0, SLIDEDP_F32, 0, 0.0};\n"
                   "  slidedp_attn_args a = {0, 1, 1, 8, 1, 1, 0, 0, 0, 0, 1.0, 0.0};\n"
                   "  slidedp_distill_args d = {0, 1, 0, SLIDEDP_BF16, 1, 1, 1.0, 1.0, 0.0};\n"
                   "  return slidedp_qk_norm_rope(0, &q, &h, &h, 0, 0, 0, 0, &h, &h, 0) != SLIDEDP_ERR_INVALID_ARG ||\n"
                   "         slidedp_attention(0, &a, &h, &h, &h, &h, 0, 0) != SLIDEDP_ERR_INVALID_ARG ||\n"
                   "         slidedp_distill_loss(0, &d, 0, 0, 0, 0, 0, 0, 0) != SLIDEDP_ERR_INVALID_ARG ||\n"
                   "         slidedp_qk_norm_rope_workspace(&q) == 0 || slidedp_attention_workspace(&a) != 0;\n}\n")
    pkg = os.path.join(root, "paper_2609_34162_b200")
    exe = tmp_path / "use"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe),
                    "-L", pkg, "-lslidedp", f"-Wl,-rpath,{pkg}"], check=True)
    subprocess.run([str(exe)], check=True)
