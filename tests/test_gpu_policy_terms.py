"""The policy loss's and the preference loss's terms on the GPU where they cancel,
vanish or are infinite, against float64.

u = 2^-24.  With a vocabulary of one, or one logit over -infinity, a row's sum of
exponentials is 1 and its log-probability exactly z - m, so nothing but the terms'
own arithmetic is off:
  * the KL term k(x) = exp(x) - x - 1: below |x| = 1/2 a series of positive weight,
    5 u of itself; from there a difference whose exp(x) - 1 is within an ulp, 2 u |exp(x)
    - 1| / k(x) <= 8.7 u (at 1/2) and its own rounding;
  * the weighted sum is float64, each result rounded once: 12 u of the mean KL term.
"""
import math

import pytest
import torch

import paper_2608_19889_amd as ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F = torch.float32
INF = float("inf")
# tokens: coefficients by each row's workgroup, by a launch before the rows, and a loss
# alone of more than 2048 tokens
COUNTS = [1, 40, 300, 3000]


def one_logit(n, vocab=1):
    """(logits, targets) of n rows whose targets have log-probability 0."""
    z = torch.full((n, vocab), -INF, device="cuda")
    z[:, 0] = torch.randn(n, device="cuda")
    return z, torch.zeros(n, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("size", [1e-7, 1e-5, 1e-3, 0.05, 0.45, 0.55, 3.0, 40.0])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("n", COUNTS)
def test_kl_term_of_any_size(n, sign, size):
    z, tg = one_logit(n)
    ref = sign * size * (0.9 + 0.2 * torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)))
    zero = torch.zeros(n, device="cuda")
    x = ref.double()
    # float64: the series where expm1(x) - x would cancel
    want = torch.where(x.abs() < 0.1, sum(x ** k / math.factorial(k) for k in range(2, 14)), torch.expm1(x) - x).mean()
    for grad in (True, False):
        for per in (False, True):
            loss, stats, _, _ = ops.policy_loss(z, tg, [0, n], zero, zero, ref, kl_coef=1.0, per_sequence=per,
                                                want_grad=grad)
            assert abs(float(stats[1]) - float(want)) <= 12 * U * float(want), (float(stats[1]), float(want))
            assert float(loss) == float(stats[1])


@pytest.mark.parametrize("n", [2, 40, 300, 3000])
def test_loss_of_advantages_that_cancel(n):
    """Normalized advantages of a policy that has not moved: the first terms are 1 and -1
    and sum to nothing, and the loss is what the KL term leaves, kl_coef times its mean.
    kl_coef is exact; 12 u as above, of values that differ by a factor of 1.2 at most."""
    z, tg = one_logit(n)
    zero = torch.zeros(n, device="cuda")
    adv = torch.ones(n, device="cuda")
    adv[1::2] = -1
    ref = -1e-3 * (1 + 0.1 * torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)))
    for grad in (True, False):
        loss, stats, _, _ = ops.policy_loss(z, tg, [0, n], zero, adv, ref, kl_coef=0.125, want_grad=grad)
        assert float(stats[0]) == 0 and float(stats[1]) > 4e-7
        # the first terms' sum: n terms of 1 / n, exact but for float64
        assert abs(float(loss) - 0.125 * float(stats[1])) <= 2 * U * float(loss) + n * 2.0 ** -53


@pytest.mark.parametrize("n", [4, 300, 3000])
def test_no_kl_coefficient_no_kl_term(n):
    """kl_coef = 0 with a reference: its mean is reported, the loss and the gradient have
    no second term, also where it is infinite (a token that the policy has ruled out)."""
    g = torch.Generator("cuda").manual_seed(n)
    z = torch.randn((n, 50), generator=g, device="cuda")
    tg = torch.randint(0, 50, (n,), generator=g, device="cuda", dtype=torch.int32)
    z[1, int(tg[1])] = -INF
    lp = ops.token_logprobs(z, tg)
    adv = torch.randn(n, generator=g, device="cuda")
    old = torch.where(torch.isfinite(lp), lp, -5.0)
    ref = torch.full((n,), -3.0, device="cuda")
    for grad in (True, False):
        want = ops.policy_loss(z, tg, [0, n], old, adv, want_grad=grad)
        got = ops.policy_loss(z, tg, [0, n], old, adv, ref, kl_coef=0.0, want_grad=grad)
        assert bool(torch.isfinite(got[0]).all()) and torch.equal(got[0], want[0])
        assert float(got[1][1]) == INF and torch.equal(got[1][::2], want[1][::2])
        assert not grad or (bool(torch.isfinite(got[3]).all()) and torch.equal(got[3], want[3]))


@pytest.mark.parametrize("n", [10, 1200])
def test_no_smoothing_no_swapped_term(n):
    """A rejected answer that the policy has ruled out (log-probability -infinity): the
    margin is infinite, its pair's loss and gradient 0 without label smoothing, the loss
    infinite with it."""
    g = torch.Generator("cuda").manual_seed(n)
    z = torch.randn((n, 50), generator=g, device="cuda")
    tg = torch.randint(0, 50, (n,), generator=g, device="cuda", dtype=torch.int32)
    cu = [0, n // 5, n // 2, n - 3, n]
    first = ops.preference_loss(z[n // 2:], tg[n // 2:], [0, n - 3 - n // 2, n - n // 2])
    z[n // 2 - 1, int(tg[n // 2 - 1])] = -INF
    for grad in (True, False):
        loss, s, u, dz = ops.preference_loss(z, tg, cu, want_grad=grad)
        assert float(s[1]) == -INF and float(u[0]) == INF
        assert abs(float(loss) - float(first[0]) / 2) <= 4 * U * float(first[0])
        if grad:
            assert not dz[:n // 2].any()
            # the other pair's: half of what it has alone, both rounded
            assert float((dz[n // 2:] - first[3] / 2).abs().max()) <= 8 * U * float(first[3].abs().max())
    assert float(ops.preference_loss(z, tg, cu, label_smoothing=0.1)[0]) == INF


# vocabularies whose logarithm lies nearly half a step between two float32 values
BETWEEN = [v for v in range(3001, 60000, 2) if abs(float(torch.tensor(math.log(v), dtype=F)) - math.log(v)) > 0.46 * 2.0 ** -20]


@pytest.mark.parametrize("n", [1, 300, 3000])
@pytest.mark.parametrize("vocab", [BETWEEN[0], BETWEEN[7]])
def test_ratio_of_a_long_row(vocab, n):
    """Rows of equal logits: the sum is exactly the vocabulary, log p = -log(vocab), and
    the loss -A q with A = 1 and q = exp(-log(vocab) - old).  log(vocab) is k log 2, held in
    two floats, and a logarithm below 0.35 within an ulp, 0.5 u; the exponential is off
    by an ulp, 2 u, its correction by the kept errors and the result by u each: 4.5 u.
    (As one float32, log(vocab) is off by 7.4 u here.)"""
    assert math.log(vocab) > 8
    z = torch.full((n, vocab), 3.25, device="cuda")
    tg = torch.arange(n, device="cuda", dtype=torch.int32) % vocab
    old = torch.full((n,), -math.log(vocab), device="cuda")
    want = -math.exp(-math.log(vocab) - float(old[0]))
    one = torch.ones(n, device="cuda")
    for grad in (True, False):
        loss = ops.policy_loss(z, tg, [0, n], old, one, want_grad=grad)[0]
        assert abs(float(loss) - want) <= 4.5 * U, ((float(loss) - want) / U, grad)
