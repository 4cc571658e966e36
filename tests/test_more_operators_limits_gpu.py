"""Block norms and policy loss where their kernels change over, exchange between blocks or are called side by side."""
import math

import pytest
import torch

from test_more_operators_gpu import BF16, F32, F64, assert_close, ctx, gen, policy_case, policy_inputs, randn, sd  # noqa: F401

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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", [(0, 0), (1, 1)])
def test_policy_rows_that_fill_a_block_of_512_threads(ctx, dtype, layout):
    """Six and eight chunks for each thread of a block that holds a row: rows that just fit, with and without the chunk more that rows off the
    16-byte grid touch, and rows one value and one chunk longer."""
    per = 16 // dtype.itemsize
    for most in (6 * 512, 8 * 512):
        for V in ((most - 1) * per, most * per - 1, most * per, most * per + 1, (most + 1) * per):
            policy_case(ctx, policy_inputs(3, V, dtype, seed=V, absent=0.0), layout=layout)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("more,layout", [(0, (0, 0)), (16, (0, 0)), (16, (3, 1)), (12345, (2, 2))])
def test_policy_rows_at_and_beyond_what_a_cluster_holds(ctx, dtype, more, layout):
    """The longest rows that are read once (1.1 MB, in eight blocks' shared memory), and longer ones: a step is then two launches, the second of
    which takes the first one's log-probabilities."""
    V = 8 * 8704 * 16 // dtype.itemsize + more
    a = policy_inputs(5, V, dtype, seed=more, absent=0.0)
    a["labels"][2] = -100                                     # absent
    a["adv"][3], a["old"][3] = 1.0, a["old"][3] - 3.0         # outside the clipped range: no gradient of the first term
    policy_case(ctx, a, layout=layout)
    policy_case(ctx, {**a, "ref": None}, layout=layout)
