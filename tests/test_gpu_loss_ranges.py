"""Rows of logits far from zero on the GPU: vocabularies masked with any finite value,
rows with a common offset, single logits near the type's largest.  The operators'
results depend on z - max(z) alone, so the bounds are those of test_gpu_losses, which
know no offset: z - m is one rounding of |z - m| u, whatever m.
"""
import math

import pytest
import torch

import paper_2608_19889_amd as ops
from test_gpu_losses import B, F, HALF, U, Rows, check, make, ref_policy, ref_preference

pytestmark = pytest.mark.gpu


def check_every_operator(z, tg, cu, losses=True):
    """Log-probabilities, their gradient and both losses, with and without a gradient,
    against float64."""
    half = HALF[z.dtype]
    r = Rows(z, tg)
    lp_bound = r.E * U + U * r.lp.abs()
    check(ops.token_logprobs(z, tg), r.lp, lp_bound, "logps")
    g = torch.Generator(device="cuda").manual_seed(61)
    rn = lambda: torch.randn(len(tg), generator=g, device="cuda")  # noqa: E731
    c = rn()
    check(ops.token_logprobs_backward(z, tg, c), r.grad(c.double()), r.grad_bound(c.double(), c.double() * 0, half),
          "dlogits")
    if not losses:
        return
    s = torch.stack([r.lp[a:b].sum() for a, b in zip(cu, cu[1:])])
    ref = (s + 4 * torch.randn(len(s), generator=g, device="cuda")).float()
    loss, dloss, s, ds, u, du, c, dc = ref_preference(r, cu, ref, 0.2, 0.1)
    for grad in (True, False):
        got = ops.preference_loss(z, tg, cu, ref, beta=0.2, label_smoothing=0.1, want_grad=grad)
        check(got[0], loss.view(1), (dloss + 4 * U * (loss + u.abs().mean() + 1)).view(1), "preference")
        check(got[1], s, ds + U * s.abs(), "seq_logps")
        check(got[2], u, du + 3 * U * u.abs(), "margins")
        if grad:
            check(got[3], r.grad(c), r.grad_bound(c, dc + 4 * U * 0.2 / len(u) * (1 + u.abs().max()), half),
                  "preference dlogits")
    moved = 0.3 * rn()
    for edge in (math.log(0.8), math.log(1.3)):  # a last digit must not decide about a whole row
        moved = torch.where((moved - edge).abs() < 2e-3, moved + 5e-3, moved)
    old, ref, adv = (r.lp - moved).float(), (r.lp + 0.3 * rn()).float(), rn()
    for per in (False, True):
        loss, dloss, stats, dstats, c, dc = ref_policy(r, cu, old, adv, ref, 0.2, 0.3, 0.1, per)
        tol = 2 * U * (2 + adv.double().abs().max())
        for grad in (True, False):
            got = ops.policy_loss(z, tg, cu, old, adv, ref, clip_low=0.2, clip_high=0.3, kl_coef=0.1, per_sequence=per,
                                  want_grad=grad)
            check(got[0], loss.view(1), (dloss + tol).view(1), "policy")
            check(got[1], stats, dstats + tol, "stats")
            check(got[2], r.lp, lp_bound, "policy logps")
            if grad:
                check(got[3], r.grad(c), r.grad_bound(c, dc + 4 * U * c.abs(), half), "policy dlogits")


MASKS = [-1e4, -65504.0, -1e6, -1e8, -1e9, -5e9, -1e10, -1e12, -1e18, -1e20, -1e30, -1e35, -1e37, -1e38, -2e38, -3e38]
# few rows (several slices each), rows by whole workgroups, and more than one workgroup's
# tokens of the loss alone
LENS = {"few": [9, 6], "many": [700, 500], "most": [1500, 700]}


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("mask", MASKS)
def test_vocabulary_masked_with_a_finite_value(mask, lens, dtype):
    """Single entries, whole groups of 8 and whole slices masked; rows of nothing but
    the mask are uniform."""
    z, tg, cu = make(LENS[lens], 9001, dtype, 60, counted=1.0)
    z[:, ::2] = mask
    z[:, 64:1024] = mask
    z[:, 3000:] = mask
    tg = torch.where(tg >= 0, tg % 900 * 2 + 1025, tg).int()
    z[3] = mask
    check_every_operator(z, tg, cu)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("offset", [1e5, -1e5, 1e6, -1e6, 1e7, -1e7, 1e20, -1e20, 3e38, -3e38])
def test_rows_with_a_common_offset(offset, lens, dtype):
    z, tg, cu = make(LENS[lens], 5003, F, 62, counted=0.8)
    check_every_operator((z + offset).to(dtype), tg, cu)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [15, 1200])
def test_a_single_large_logit(n, dtype):
    """Beside one logit of 3e38 nothing else has a probability; a target there has
    log-probability 0, one elsewhere the difference."""
    z, tg, cu = make([n - n // 2, n // 2], 9001, dtype, 63, counted=1.0)
    z[:, 4000] = 3e38
    check_every_operator(z, tg, cu, losses=False)
    tg = torch.where(tg >= 0, 4000, tg).int()
    check_every_operator(z, tg, cu)


@pytest.mark.parametrize("tokens", [128, 1000])
def test_errors_of_many_rows_do_not_add_up(tokens):
    """A sequence's log-probability adds up its tokens' errors, so they must not share a
    sign: their mean over 4000 rows and more is at most half a step, u / 2.  (Single rows
    are off by about 1 u, their mean by 1 / sqrt(4000) of that by chance.)  Each row is a
    pair's chosen sequence, its reference the exact value rounded to float32: the margin
    is the error and what that rounding left, in full."""
    g = torch.Generator(device="cuda").manual_seed(64)
    cu = [0] + [t + 1 for t in range(tokens) for _ in range(2)]
    errors = []
    for _ in range(-(-4096 // tokens)):
        z = 2 * torch.randn(tokens, 32000, generator=g, device="cuda")
        tg = z.argmax(-1).int()
        lp = torch.log_softmax(z.double(), -1).gather(1, tg.long()[:, None])[:, 0]
        ref = torch.zeros(2 * tokens, device="cuda")
        ref[::2] = lp.float()
        margins = ops.preference_loss(z, tg, cu, ref, beta=1.0, want_grad=False)[2]
        errors.append(margins.double() - (lp - ref[::2].double()))
    errors = torch.cat(errors)
    assert float(errors.abs().max()) <= 12 * U and abs(float(errors.mean())) <= U / 2, float(errors.mean()) / U
