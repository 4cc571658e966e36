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


# Forms that take each of the kernels: rows held by a warp, by a block, in shared memory of one block and of a cluster, and in none.
KERNELS = [(12, 1000), (12, 20000), (170, 40000), (12, 70001), (4, 600003)]


def confident(N, V, dtype, seed):
    """Labels that have all but 1e-2 to 1e-13 of their rows' probability, advantages without an old policy (the ratio is one)."""
    g = gen(seed)
    z = randn(g, N, V, dtype=dtype)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    labels[0], labels[-1] = 0, V - 1
    lack = torch.linspace(2.0, 13.0, N, device="cuda", dtype=F64)[torch.randperm(N, generator=g, device="cuda")] * math.log(10.0)
    others = z.double().scatter(1, labels[:, None], -math.inf).logsumexp(1)
    z.scatter_(1, labels[:, None], (others + lack).to(dtype)[:, None])
    return z, labels.to(torch.int32), randn(g, N), randn(g, N)


@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V", KERNELS)
def test_policy_of_tokens_that_are_all_but_certain(ctx, dtype, N, V, tau):
    """What the label's probability lacks of one keeps its digits, however little it is: log-probability and gradient are off by 2e-5 of
    themselves (the tolerance of a probability in more_operators_ref.policy) and their own rounding, and a row's gradient adds up to zero to within
    twice that."""
    z, labels, adv, gr = confident(N, V, dtype, seed=V)
    z = (z.double() * tau).to(dtype)
    at = labels.long()[:, None]
    zd = z.double() / tau
    t = zd.gather(1, at)[:, 0] - zd.scatter(1, at, -math.inf).logsumexp(1)       # the label's log odds
    lp, rest = -torch.log1p(torch.exp(-t)), 1.0 / (1.0 + torch.exp(t))
    f = -(adv * gr).double()[:, None] / tau                                      # d loss / d logp = -adv
    want = f * (torch.zeros_like(zd).scatter(1, at, 1.0) - torch.log_softmax(zd, 1).exp())
    want.scatter_(1, at, f * rest[:, None])
    new = lambda: torch.empty(N, device="cuda")  # noqa: E731
    loss, logp, logp2, dz, dz2 = new(), new(), new(), torch.empty_like(z), torch.empty_like(z)
    ctx.slidedp_policy_loss(z, labels, None, None, adv, loss, logp, temperature=tau)
    ctx.slidedp_policy_loss_backward(z, labels, None, None, adv, logp, gr, dz, temperature=tau)
    ctx.slidedp_policy_step(z, labels, None, None, adv, gr, loss, logp2, dz2, temperature=tau)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    for what, p, d in (("two calls", logp, dz), ("step", logp2, dz2)):
        assert_close(what + ": logp", p, lp, 2e-5 * lp.abs())
        assert_close(what + ": dz", d, want, (2e-5 + half) * want.abs() + 1e-37)
        if dtype == F32:
            assert_close(what + ": sum", d.double().sum(1), torch.zeros_like(lp), (4e-5 + 2 * half) * want.gather(1, at)[:, 0].abs() + V * 1e-37)


def test_policy_second_term_near_the_reference(ctx):
    """e^k - k - 1 is k^2 / 2 there: off by the digits of k, not of k / k^2. The log-probabilities are close to zero, so that FP32 has
    k's digits: 2e-5 of logp beside k, up to three times that in the term, and four roundings."""
    z, labels, _, _ = confident(64, 1000, F32, seed=3)
    at = labels.long()[:, None]
    t = z.double().gather(1, at)[:, 0] - z.double().scatter(1, at, -math.inf).logsumexp(1)
    lp = -torch.log1p(torch.exp(-t))
    for size in (3e-3, 0.1, 0.9, 1.1, 3.0):
        for sign in (-1.0, 1.0):
            refp = (lp + sign * size).float()
            k = refp.double() - lp
            exact = torch.where(k.abs() < 0.01, k * k * (0.5 + k / 6 + k * k / 24 + k ** 3 / 120), torch.expm1(k) - k)
            loss, logp = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
            ctx.slidedp_policy_loss(z, labels, None, refp, None, loss, logp, kl_weight=2.0)
            tol = exact * (2.0 ** -21 + 3 * 2e-5 * lp.abs() / k.abs() * torch.clamp(k.abs(), min=1.0))
            assert_close(f"loss {sign * size}", loss, 2.0 * exact, 2.0 * tol)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V", KERNELS)
def test_policy_tokens_without_probability(ctx, dtype, N, V):
    """A label whose logit is -inf, others being finite: logp is -inf, and the second term's limit is +inf, not NaN."""
    z = randn(gen(V), N, V, dtype=dtype)
    labels = (torch.arange(N, device="cuda") * 31 % V).to(torch.int32)
    z.scatter_(1, labels.long()[:, None], -math.inf)
    f = torch.zeros(N, device="cuda")
    loss, logp, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
    for call in (lambda: ctx.slidedp_policy_loss(z, labels, None, f, None, loss, logp, kl_weight=0.1),
                 lambda: ctx.slidedp_policy_step(z, labels, None, f, None, None, loss, logp, dz, kl_weight=0.1)):
        loss.fill_(0.0), logp.fill_(0.0)
        call()
        assert (logp == -math.inf).all() and (loss == math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V", KERNELS + [(700, 9000)])
def test_policy_backward_of_very_unlikely_tokens(ctx, dtype, N, V):
    """Labels whose log-probability is anything down to -inf, rows far from zero among them: the gradient's probabilities are off by 2e-5 of
    themselves (as in more_operators_ref.policy), not by 2^-24 of the log-probability that the forward call has saved."""
    g = gen(V + 1)
    z = randn(g, N, V, dtype=dtype)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    labels[0], labels[-1] = 0, V - 1
    row = torch.arange(N, device="cuda")
    z[row % 6 == 5] += 3e6 if dtype == F32 else 512.0
    down = torch.tensor([-40.0, -90.0, -700.0, -3e4, -math.inf, -9e5 if dtype == F32 else -2e4], device="cuda")[row % 6]
    z[row, labels] = (z[row, labels].double() + down).to(dtype)
    adv, gr = randn(g, N), randn(g, N)
    p = torch.log_softmax(z.double(), 1).exp()
    want = (-(adv * gr)).double()[:, None] * (torch.zeros_like(p).scatter(1, labels[:, None], 1.0) - p)
    labels = labels.to(torch.int32)
    logp, loss, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
    ctx.slidedp_policy_loss(z, labels, None, None, adv, loss, logp)
    ctx.slidedp_policy_loss_backward(z, labels, None, None, adv, logp, gr, dz)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    tol = (2e-5 + half) * want.abs() + 1e-37
    assert_close("dz", dz, want, tol)
    step, logp2 = torch.empty_like(z), torch.empty_like(logp)       # its log-probabilities may differ in the last bits: the saved ones stay
    ctx.slidedp_policy_step(z, labels, None, None, adv, gr, loss, logp2, step)
    assert_close("step: dz", step, want, tol)
    ctx.slidedp_policy_loss_backward(z, labels, None, None, adv, logp, gr, z)                 # in place
    assert torch.equal(z, dz)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V", KERNELS + [(700, 9000)])
def test_policy_labels_whose_logit_is_no_number(ctx, dtype, N, V):
    """NaN and +inf at the label, or a row of -inf: log-probability and gradient are NaN in that row, and the other rows' bits are
    what they are without it. A row of one finite logit among -inf is certain of it."""
    g = gen(V + 2)
    z = randn(g, N, V, dtype=dtype)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    adv, gr = randn(g, N), randn(g, N)

    def run(z):
        out = []
        for step in (False, True):
            loss, logp, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
            if step:
                ctx.slidedp_policy_step(z, labels32, None, None, adv, gr, loss, logp, dz)
            else:
                ctx.slidedp_policy_loss(z, labels32, None, None, adv, loss, logp)
                ctx.slidedp_policy_loss_backward(z, labels32, None, None, adv, logp, gr, dz)
            out.append((loss, logp, dz))
        return out

    labels32 = labels.to(torch.int32)
    clean = run(z)
    bad = z.clone()
    bad[0, labels[0]], bad[1, labels[1]], bad[2] = math.nan, math.inf, -math.inf
    bad[3] = -math.inf
    bad[3, labels[3]] = 1.5
    keep = torch.arange(N, device="cuda") > 3
    for (loss, logp, dz), (l0, p0, d0) in zip(run(bad), clean):
        assert logp[:3].isnan().all() and dz[:3].isnan().all()
        assert logp[3] == 0 and not dz[3].any()
        assert torch.equal(loss[keep], l0[keep]) and torch.equal(logp[keep], p0[keep]) and torch.equal(dz[keep], d0[keep])
