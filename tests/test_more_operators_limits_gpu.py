"""Block norms and policy loss where their kernels change over, exchange between blocks or are called side by side."""
import math

import pytest
import torch

from test_more_operators_gpu import BF16, F32, F64, assert_close, ctx, gen, policy_inputs, randn, sd  # noqa: F401

pytestmark = pytest.mark.gpu


def exact_logp(z, labels, tau=1.0):
    """In 64 bits; 0 for absent rows."""
    has = (labels >= 0) & (labels < z.shape[1])
    lp = torch.log_softmax(z.double() / tau, 1).gather(1, labels.clamp(0, z.shape[1] - 1).long()[:, None])[:, 0]
    return torch.where(has, lp, 0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V", [(1, 16384), (3, 65537), (40, 131072), (150, 16391), (296, 40000), (591, 8200)])
def test_policy_forward_of_rows_that_blocks_share(ctx, dtype, N, V):
    """Clusters of two, four and eight blocks to a row, with absent rows among them, again and again. The tolerance is that of
    more_operators_ref.policy."""
    a = policy_inputs(N, V, dtype, seed=N, absent=0.3)
    want = exact_logp(a["z"], a["labels"])
    for _ in range(5):
        lp = torch.full((N,), 9.0, device="cuda")
        ctx.slidedp_policy_loss(a["z"], a["labels"], None, None, None, None, lp)
        assert_close("logp", lp, want, 5e-6 + 2.0 ** -22 * want.abs())


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_norm_sums_without_tokens_are_zeros_whatever_the_gate_holds(ctx, dtype, sigmoid):
    H = 70
    x = torch.empty(0, H, dtype=dtype, device="cuda")
    ws = torch.empty(ctx.slidedp_block_norm_workspace(x), dtype=torch.uint8, device="cuda")
    for bad in (math.inf, math.nan):
        w, gate = torch.full((H,), bad, dtype=dtype, device="cuda"), torch.full((H,), bad, dtype=dtype, device="cuda")
        sums = [torch.full((H,), 5.0, device="cuda") for _ in range(3)]
        ctx.slidedp_block_norm_backward(x, x, w, gate, w, x, x, x, x, *sums, ws, gate_sigmoid=sigmoid)
        assert not any(s.any() for s in sums)
