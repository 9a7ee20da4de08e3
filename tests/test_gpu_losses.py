"""Log-probabilities of tokens, the preference loss and the clipped policy loss on
the GPU, against float64.

u = 2^-24 (half a step of float32), h half a step of the gradient's type (float32 u,
bf16 2^-8).  Row by row, with x_v = z_v - m (m the row's maximum):
  * exp(x) is off by (3 |x| + 4) u of itself: the subtraction's rounding, the product
    with log2 e and its constant (each |x| u at most in the exponent), the hardware
    exponential (an ulp, 2 u) and the result's rescaling;
  * S = sum exp(x) by E u of itself, E = the additions in a row (V / 256 of a thread's
    share and 64 to join them) + the mean of 3 |x| + 4 under the probabilities; log S
    by E u;
  * lp (float64 from there) by E u, and by u |lp| as a float32 output;
  * a loss is off by its derivatives times E u; the coefficient c = dloss / dlp of a
    token by |dc / dlp| E u + 2 u |c|;
  * dz = c ([v = y] - p_v) by |c| p ((3 |x| + 6) + E) u + 3 u |c| at the target + what
    c is off by, and its own rounding h |dz|.
"""
import math

import numpy as np
import pytest
import torch

import paper_2608_19889_amd as ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16
HALF = {F: U, B: 2.0 ** -8}
INF = float("inf")


def make(lens, V, dtype, seed, ld=None, counted=0.7, spread=2.0):
    """(logits, targets, cu) with some positions that do not count; the last of every
    sequence never does."""
    T = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((T, ld or V), float("nan"), device="cuda", dtype=dtype)
    tg = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    z = torch.randn((T, V), generator=g, device="cuda") * spread
    if T:
        z[torch.arange(T), tg.long()] += 8 * torch.rand((T,), generator=g, device="cuda")
    wide[:, :V] = z
    off = torch.rand((T,), generator=g, device="cuda") > counted
    cu = np.cumsum([0, *lens]).tolist()
    off[[e - 1 for a, e in zip(cu, cu[1:]) if e > a]] = True
    tg[off] = torch.where(torch.rand((T,), generator=g, device="cuda") < 0.5, -1, V + 5)[off].int()
    return wide[:, :V], tg, cu


class Rows:
    """Everything of the rows in float64, and the bounds above."""

    def __init__(self, z, tg):
        V = z.shape[1]
        zd = z.double()
        self.ok = (tg >= 0) & (tg < V)
        self.at = tg.long().clamp(0, V - 1)
        self.x = zd - zd.amax(-1, keepdim=True)
        self.p = torch.softmax(zd, -1)
        lp = torch.log_softmax(zd, -1)[torch.arange(len(tg)), self.at]
        self.lp = torch.where(self.ok, lp, 0.0)
        far = torch.where(self.p > 0, self.x.abs(), 0.0)
        self.far = far
        self.E = torch.where(self.ok, V / 256 + 64 + (self.p * (3 * far + 4)).sum(-1), 0.0)

    def grad(self, c):
        c = torch.where(self.ok, c, 0.0)
        g = -c[:, None] * self.p
        g[torch.arange(len(c)), self.at] += c
        return torch.where(self.ok[:, None], g, 0.0)

    def grad_bound(self, c, dc, half):
        """of dz for coefficients c that are off by dc"""
        c, dc = (torch.where(self.ok, v, 0.0)[:, None].abs() for v in (c, dc))
        one = torch.zeros_like(self.p)
        one[torch.arange(len(c)), self.at] = 1
        return (c * self.p * (3 * self.far + 6 + self.E[:, None]) * U + 3 * U * c * one + dc * (one + self.p)
                + half * self.grad(c[:, 0]).abs() + 1e-42)


def check(got, ref, bound, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((off / bound.clamp_min(1e-300)).max()))


def ref_preference(r, cu, ref, beta, e):
    s = torch.stack([r.lp[a:b].sum() for a, b in zip(cu, cu[1:])])
    ds = torch.stack([r.E[a:b].sum() for a, b in zip(cu, cu[1:])]) * U
    d = (s - (ref.double() if ref is not None else 0)).view(-1, 2)
    u, du = beta * (d[:, 0] - d[:, 1]), beta * ds.view(-1, 2).sum(-1)
    yes, no = torch.sigmoid(u), torch.sigmoid(-u)
    loss = -((1 - e) * torch.nn.functional.logsigmoid(u) + e * torch.nn.functional.logsigmoid(-u))
    k = beta / len(u)
    slope = k * (e * yes - (1 - e) * no)
    c = torch.zeros_like(r.lp)
    dc = torch.zeros_like(r.lp)
    for j, (a, b) in enumerate(zip(cu, cu[1:])):
        c[a:b] = slope[j // 2] * (1 if j % 2 == 0 else -1)
        dc[a:b] = k * 0.25 * du[j // 2] + 2 * U * slope[j // 2].abs()
    return loss.mean(), du.mean(), s, ds, u, du, c, dc


def ref_policy(r, cu, old, adv, ref, lo, hi, kl, per):
    ok = r.ok
    w = torch.zeros_like(r.lp)
    if per:
        full = [(a, b) for a, b in zip(cu, cu[1:]) if bool(ok[a:b].any())]
        for a, b in full:
            w[a:b] = 1.0 / (int(ok[a:b].sum()) * len(full))
    else:
        w[:] = 1.0 / max(1, int(ok.sum()))
    w = torch.where(ok, w, 0.0)
    old, adv, rf = (torch.where(ok, v.double(), 0.0) if v is not None else r.lp for v in (old, adv, ref))
    q = torch.exp(r.lp - old)
    stop = ((adv > 0) & (q > 1 + hi)) | ((adv < 0) & (q < 1 - lo))
    term = -adv * torch.where(stop, q.clamp(1 - lo, 1 + hi), q)
    term = torch.where(adv == 0, 0.0, term)
    g = rf - r.lp
    k3 = torch.expm1(g) - g
    c = w * (torch.where(stop | (adv == 0), 0.0, -adv * q) - kl * torch.expm1(g))
    e = r.E * U
    dl = torch.where(stop | (adv == 0), 0.0, (adv * q).abs()) + kl * torch.expm1(g).abs()
    dc = w * (torch.where(stop | (adv == 0), 0.0, (adv * q).abs()) + kl * torch.exp(g)) * e + 2 * U * c.abs()
    stats = torch.stack([(w * term).sum(), (w * k3).sum(), (w * stop).sum()])
    dstats = torch.stack([(w * (adv * q).abs().nan_to_num(0, 0, 0) * e).sum(), (w * torch.expm1(g).abs() * e).sum(),
                          torch.zeros((), dtype=torch.float64, device=w.device)])
    return (w * (term + kl * k3)).sum(), (w * dl * e).sum(), stats, dstats, c, dc


# lengths, vocabulary, row stride, type: one token; a vocabulary of one; sequences
# without a position; each edge of a slice (2048), of a gradient slice (8192); rows
# of odd length at any alignment; many slices a row, and whole rows
CASES = [([2, 1], 1, 1, F), ([1, 1], 2, 2, B), ([5, 0, 0, 3], 7, 9, B), ([9, 4], 50, 50, F), ([20, 13], 2047, 2047, F),
         ([20, 13], 2048, 2048, B), ([20, 13], 2049, 2056, B), ([3, 4, 5, 6], 8191, 8192, B), ([7, 7], 8193, 8193, F),
         ([11, 30], 50257, 50257, B), ([11, 30], 50257, 50272, F), ([100, 87, 33, 160], 32000, 32000, B),
         ([600, 400, 90, 300], 5003, 5003, F), ([1100, 1200], 4100, 4100, B)]
# each width that a workgroup holds in registers (4 groups of 8 a thread, then 64
# registers of 256, 512 and 1024 threads, then more), and rows longer than that
LONG = [([600, 0, 425], 2050, 2050, F), ([1024], 8192, 8192, B), ([700, 330], 8197, 8200, F),
        ([500, 1, 530], 16385, 16385, F), ([1030], 32771, 32771, B), ([515, 515], 40003, 40003, F),
        ([1025], 65544, 65544, B), ([300, 730], 70001, 70001, F), ([1026], 131072, 131072, B),
        ([1027], 140003, 140005, B)]
name = lambda c: "%dx%d-%s" % (sum(c[0]), c[1], "f32" if c[3] == F else "bf16")  # noqa: E731


@pytest.mark.parametrize("case", CASES + LONG, ids=name)
def test_log_probabilities_and_their_gradient(case):
    lens, V, ld, dtype = case
    z, tg, cu = make(lens, V, dtype, 1, ld)
    r = Rows(z, tg)
    got = ops.token_logprobs(z, tg)
    check(got, r.lp, r.E * U + U * r.lp.abs(), "logps")
    assert not got[~r.ok].any()
    c = torch.randn(len(tg), device="cuda")
    c[~r.ok] = float("nan")
    g = ops.token_logprobs_backward(z, tg, c)
    assert g.dtype == dtype
    check(g, r.grad(c.double()), r.grad_bound(c.double(), c.double() * 0, HALF[dtype]), "dlogits")
    # the other type, in rows of another stride whose last columns stay as they were
    other = B if dtype == F else F
    wide = torch.full((len(tg), V + 3), 5.0, device="cuda", dtype=other)
    ops.token_logprobs_backward(z, tg, c, dlogits=wide[:, :V])
    check(wide[:, :V], r.grad(c.double()), r.grad_bound(c.double(), c.double() * 0, HALF[other]), "dlogits")
    assert (wide[:, V:] == 5).all()


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
@pytest.mark.parametrize("case", CASES, ids=name)
def test_preference_loss(case, smoothing):
    lens, V, ld, dtype = case
    z, tg, cu = make(lens, V, dtype, 2, ld)
    r = Rows(z, tg)
    g = torch.Generator(device="cuda").manual_seed(3)
    s = torch.stack([r.lp[a:b].sum() for a, b in zip(cu, cu[1:])])
    for ref in ((s + 4 * torch.randn(len(lens), generator=g, device="cuda")).float(), None):
        beta = 0.2 if ref is not None else 0.01
        loss, dloss, s, ds, u, du, c, dc = ref_preference(r, cu, ref, beta, smoothing)
        got = ops.preference_loss(z, tg, cu, ref, beta=beta, label_smoothing=smoothing)
        # beta and e reach the kernel as float32: u of each
        check(got[0], loss.view(1), (dloss + 4 * U * (loss + u.abs().mean() + 1)).view(1), "loss")
        check(got[1], s, ds + U * s.abs(), "seq_logps")
        check(got[2], u, du + 3 * U * u.abs(), "margins")
        check(got[3], r.grad(c), r.grad_bound(c, dc + 4 * U * beta / len(u) * (1 + u.abs().max()), HALF[dtype]),
              "dlogits")
        only = ops.preference_loss(z, tg, cu, ref, beta=beta, label_smoothing=smoothing, want_grad=False)
        assert only[3] is None and all(torch.equal(a, b) for a, b in zip(only[:3], got))


@pytest.mark.parametrize("per", [False, True])
@pytest.mark.parametrize("case", CASES + LONG, ids=name)
def test_policy_loss(case, per):
    lens, V, ld, dtype = case
    z, tg, cu = make(lens, V, dtype, 4, ld)
    r = Rows(z, tg)
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda: torch.randn(len(tg), generator=g, device="cuda")  # noqa: E731
    moved = 0.3 * rn()
    for edge in (math.log(0.8), math.log(1.3)):  # a last digit must not decide about a whole row
        moved = torch.where((moved - edge).abs() < 1e-3, moved + 3e-3, moved)
    old, ref, adv = (r.lp - moved).float(), (r.lp + 0.3 * rn()).float(), rn()
    adv[::7] = 0
    for v in (old, ref, adv):
        v[~r.ok] = float("nan")
    for rf, kl in ((ref, 0.1), (ref, 0.0), (None, 0.0)):
        loss, dloss, stats, dstats, c, dc = ref_policy(r, cu, old, adv, rf, 0.2, 0.3, kl, per)
        got = ops.policy_loss(z, tg, cu, old, adv, rf, clip_low=0.2, clip_high=0.3, kl_coef=kl, per_sequence=per)
        # the clip bounds and kl_coef reach the kernel as float32
        tol = 2 * U * (1 + (adv.double().abs().nan_to_num(0).max() + 1))
        check(got[0], loss.view(1), (dloss + tol).view(1), "loss")
        check(got[1], stats, dstats + tol, "stats")
        check(got[2], r.lp, r.E * U + U * r.lp.abs(), "logps")
        check(got[3], r.grad(c), r.grad_bound(c, dc + 4 * U * c.abs(), HALF[dtype]), "dlogits")
        only = ops.policy_loss(z, tg, cu, old, adv, rf, clip_low=0.2, clip_high=0.3, kl_coef=kl, per_sequence=per,
                               want_grad=False)
        assert only[3] is None
        check(only[0], loss.view(1), (dloss + tol).view(1), "loss alone")
        check(only[1], stats, dstats + tol, "stats alone")
        check(only[2], r.lp, r.E * U + U * r.lp.abs(), "logps alone")


# more sequences than a workgroup keeps the boundaries of (1024); as many tokens as a
# workgroup counts by itself (256) and one more; few tokens in many sequences
MANY = [([1, 0, 2] * 400, 130, 130, F), ([64, 0, 0, 192], 301, 301, B), ([200, 0, 0, 57], 300, 300, F),
        ([1, 0, 0, 0] * 80, 41, 41, B), ([0, 65, 0, 1] * 3 + [0, 0], 9000, 9000, F),
        # pairs whose workgroups work out the coefficients, up to 128 tokens and 256 sequences, and past it
        ([1, 0] * 128, 2500, 2501, B), ([1, 0] * 127 + [0, 0, 1, 0], 2049, 2049, F), ([50, 78], 65536, 65536, B),
        ([50, 78], 65537, 65537, B), ([100, 28], 1003, 1003, F)]


@pytest.mark.parametrize("case", MANY, ids=name)
def test_many_sequences(case):
    test_preference_loss(case, 0.1)
    test_policy_loss(case, False)
    test_policy_loss(case, True)


def test_what_the_binding_refuses():
    z, tg, cu = make([4, 5], 30, F, 50)
    f = torch.zeros(9, device="cuda")
    for text, call in (
            ("int32", lambda: ops.token_logprobs(z, tg.long())),
            ("targets must hold 9", lambda: ops.token_logprobs(z, tg[:8])),
            ("bfloat16 or float32", lambda: ops.token_logprobs(z.half(), tg)),
            ("tensors on", lambda: ops.token_logprobs(z, tg.cpu())),
            ("dlogps", lambda: ops.token_logprobs_backward(z, tg, f.double())),
            ("dlogits must", lambda: ops.token_logprobs_backward(z, tg, f, dlogits=torch.empty(9, 31, device="cuda"))),
            ("contiguous columns", lambda: ops.token_logprobs_backward(
                z, tg, f, dlogits=torch.empty(30, 9, device="cuda").t())),
            ("pairs", lambda: ops.preference_loss(z, tg, [0, 9])),
            ("pairs", lambda: ops.preference_loss(z, tg, [0, 2, 4, 9])),
            ("ref_logps", lambda: ops.preference_loss(z, tg, cu, f)),
            ("cu_device", lambda: ops.preference_loss(z, tg, cu, cu_device=tg[:2])),
            ("old_logps", lambda: ops.policy_loss(z, tg, cu, f[:3], f))):
        with pytest.raises(ValueError, match=text):
            call()
    from paper_2608_19889_amd import AxonError
    with pytest.raises(AxonError, match="end at 8"):
        ops.preference_loss(z, tg, [0, 4, 8])
    with pytest.raises(AxonError, match="logits' buffer"):
        wide = torch.empty(9, 64, device="cuda")
        ops.token_logprobs_backward(wide[:, :30], tg, f, dlogits=wide.view(18, 32)[:9, :30])
    # layouts that the kernels do not take are copied: a transposed input, a broadcast row
    want = ops.token_logprobs(z, tg)
    assert torch.equal(ops.token_logprobs(z.t().contiguous().t(), tg), want)
    assert torch.equal(ops.token_logprobs(z[:1].expand(9, 30), tg), ops.token_logprobs(z[:1].repeat(9, 1), tg))


def test_nothing_counts():
    """Every position masked: loss, statistics and gradients 0, whatever the rows
    hold; sequences without a counted position beside one that has some."""
    z = torch.full((6, 40), float("nan"), device="cuda")
    tg = torch.full((6,), -1, dtype=torch.int32, device="cuda")
    nan = torch.full((6,), float("nan"), device="cuda")
    assert not ops.token_logprobs(z, tg).any()
    assert not ops.token_logprobs_backward(z, tg, nan).any()
    for per in (False, True):
        got = ops.policy_loss(z, tg, [0, 2, 2, 6], nan, nan, nan, kl_coef=0.1, per_sequence=per)
        assert all(not v.any() for v in got)
    loss, s, u, dz = ops.preference_loss(z, tg, [0, 2, 6])
    assert abs(float(loss) - math.log(2)) < 1e-6 and not s.any() and not u.any() and not dz.any()
    # one counted position in the last sequence: its weight is 1 either way
    z[5] = 0.0
    tg[5] = 3
    nan[5] = 0.0
    old = nan - math.log(40)
    adv = torch.where(nan == 0, 2.0, nan)
    for per in (False, True):
        got = ops.policy_loss(z, tg, [0, 2, 2, 6], old, adv, per_sequence=per)
        assert abs(float(got[0]) + 2) < 1e-5 and not got[3][:5].any() and abs(float(got[3][5, 3]) + 2 * 39 / 40) < 1e-5
    # no rows at all
    e = torch.empty(0, 40, device="cuda")
    n = torch.empty(0, dtype=torch.int32, device="cuda")
    f = torch.empty(0, device="cuda")
    assert ops.token_logprobs(e, n).shape == (0,) and ops.token_logprobs_backward(e, n, f).shape == (0, 40)
    assert float(ops.policy_loss(e, n, [0, 0], f, f)[0]) == 0
    assert abs(float(ops.preference_loss(e, n, [0, 0, 0])[0]) - math.log(2)) < 1e-6


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[9, 6], [900, 300]], ids=["few", "many"])
def test_masked_vocabulary(lens, dtype):
    """Tokens ruled out by -infinity or the type's lowest value have probability and
    gradient 0, also where whole slices of a row hold nothing else; rows of nothing but
    the lowest value are uniform."""
    n = sum(lens)
    z, tg, cu = make(lens, 9001, dtype, 6, counted=1.0)
    for i, low in enumerate((-INF, torch.finfo(dtype).min)):
        z[:, 3000:] = low
        z[:, ::2] = low
        tg = torch.where(tg >= 0, tg % 1500 * 2 + 1, tg).int()
        r = Rows(z, tg)
        check(ops.token_logprobs(z, tg), r.lp, r.E * U + U * r.lp.abs(), "logps")
        c = torch.ones(n, device="cuda")
        g = ops.token_logprobs_backward(z, tg, c)
        assert not g[:, 3000:].any() and not g[:, ::2].any()
        check(g, r.grad(c.double()), r.grad_bound(c.double(), c.double() * 0, HALF[dtype]), "dlogits")
    # a target that is ruled out: log-probability -inf, and a gradient that is the formula's
    z[0, 1] = -INF
    tg[0] = 1
    assert float(ops.token_logprobs(z, tg)[0]) == -INF
    g = ops.token_logprobs_backward(z, tg, torch.ones(n, device="cuda"))
    assert float(g[0, 1]) == 1 and bool(torch.isfinite(g).all())
    z[2] = torch.finfo(dtype).min
    tg[2] = 5
    assert abs(float(ops.token_logprobs(z, tg)[2]) + math.log(9001)) < 1e-5
    g = ops.token_logprobs_backward(z, tg, torch.ones(n, device="cuda"))[2].double()
    assert abs(float(g[5]) - 1) < 2.0 ** -8 and abs(float(g[7]) * 9001 + 1) < 2.0 ** -7


@pytest.mark.parametrize("n", [40, 1100])
def test_not_a_number_stays_in_its_row(n):
    z, tg, _ = make([n], 3000, F, 7, counted=1.0)
    z[3, 77] = float("nan")
    z[8, 2999] = INF
    got = ops.token_logprobs(z, tg)
    assert got[3].isnan() and got[8].isnan() and int((~torch.isfinite(got)).sum()) == 2
    g = ops.token_logprobs_backward(z, tg, torch.ones(n, device="cuda"))
    bad = ~torch.isfinite(g).all(-1)
    assert bad.nonzero().flatten().tolist() == [3, 8]


def test_ratio_that_overflows():
    """A token that the sampling policy gave next to no probability: with A > 0 the
    clipped value holds, with A = 0 there is no term, with A < 0 the loss is infinite
    by its formula."""
    z, tg, _ = make([4], 30, F, 8, counted=1.0)
    old = torch.full((4,), -3e38, device="cuda")
    adv = torch.tensor([2.0, 0.0, 1.0, 5.0], device="cuda")
    loss, stats, _, dz = ops.policy_loss(z, tg, [0, 4], old, adv, clip_high=0.5)
    assert abs(float(loss) + 3 * 1.5 / 3) < 1e-5 and abs(float(stats[2]) - 2 / 3) < 1e-6 and not dz.any()
    adv[0] = -1
    assert float(ops.policy_loss(z, tg, [0, 4], old, adv)[0]) == INF


def test_gradient_in_the_logits_buffer():
    """dlogits in place of the logits gives the same bits; what lies between the rows
    keeps its own."""
    for dtype, lens in ((F, [30, 50]), (B, [30, 50]), (F, [700, 600]), (B, [700, 600])):
        z, tg, cu = make(lens, 10007, dtype, 9, 10012)
        r = Rows(z, tg)
        ref = torch.randn(sum(lens), device="cuda") + r.lp.float()
        want = ops.policy_loss(z, tg, cu, ref, ref, ref, kl_coef=0.1)
        base = z._base
        between = base[:, 10007:].clone()
        got = ops.policy_loss(z, tg, cu, ref, ref, ref, kl_coef=0.1, dlogits=z)
        assert got[3] is z and all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(base[:, 10007:].view(torch.int16), between.view(torch.int16))


@pytest.mark.parametrize("ld", [10007, 10012])
@pytest.mark.parametrize("lens", [[30, 50], [100, 0, 60, 40], [700, 600]], ids=["few", "some", "many"])
@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_other_gradients_in_the_logits_buffer(dtype, lens, ld):
    z, tg, cu = make(lens, 10007, dtype, 12, ld)
    c = torch.randn(sum(lens), device="cuda")
    for call in (lambda out: ops.preference_loss(z, tg, cu, dlogits=out),
                 lambda out: (ops.token_logprobs_backward(z, tg, c, dlogits=out),)):
        keep = z.clone()
        want = call(torch.empty_like(z))
        got = call(z)
        assert got[-1] is z and all(torch.equal(a, b) for a, b in zip(got, want))
        z.copy_(keep)


def test_gradients_against_differences():
    """The slope of each loss along a direction v of unit entries, by central
    differences of the kernel's own forward (step 2^-7): the third derivative of a sum
    of log-probabilities along v is at most about 10 per row, and float32 leaves u times
    the loss's terms over the step."""
    lens, V = [9, 12, 7, 10], 60
    z, tg, cu = make(lens, V, F, 10)
    r = Rows(z, tg)
    g = torch.Generator(device="cuda").manual_seed(11)
    v = torch.randn((38, V), generator=g, device="cuda")
    old = (r.lp + 0.05 * torch.randn(38, generator=g, device="cuda")).float()
    adv = torch.randn(38, generator=g, device="cuda")
    ref = torch.tensor([-30.0, -28.0, -20.0, -25.0], device="cuda")
    h = 2.0 ** -7
    # wide clip bounds: the slope of a clipped loss jumps at its edge
    for f, rows in ((lambda x: ops.preference_loss(x, tg, cu, ref, beta=0.3, label_smoothing=0.1), 3.0),
                    (lambda x: ops.policy_loss(x, tg, cu, old, adv, old, clip_low=0.9, clip_high=3.0, kl_coef=0.2,
                                               per_sequence=True), 4.0)):
        slope = float((f(z)[3].double() * v.double()).sum())
        diff = (float(f(z + h * v)[0]) - float(f(z - h * v)[0])) / (2 * h)
        assert abs(slope - diff) <= 10 * rows * h * h / 6 * 10 + 16 * U * rows / h, (slope, diff)


def _policy_inputs(lens, V, dtype, seed):
    z, tg, cu = make(lens, V, dtype, seed)
    lp = ops.token_logprobs(z, tg)
    n = torch.randn(3, len(tg), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + 1))
    return z, tg, cu, torch.tensor(cu, dtype=torch.int32, device="cuda"), lp + 0.2 * n[0], n[1], lp + 0.2 * n[2]


def test_two_streams_at_once():
    """Calls that overlap on two streams, each with the workspace its own call makes."""
    a, b = _policy_inputs([300, 200], 20011, F, 12), _policy_inputs([100, 333], 30011, B, 14)
    call = lambda i, st: ops.policy_loss(i[0], i[1], i[2], i[4], i[5], i[6], kl_coef=0.1, per_sequence=True,  # noqa: E731
                                         cu_device=i[3], stream=st)
    want = [call(a, None), call(b, None)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = [(call(a, s1), call(b, s2)) for _ in range(6)]
    torch.cuda.synchronize()
    for x, y in got:
        assert all(torch.equal(p, q) for p, q in zip(x, want[0]))
        assert all(torch.equal(p, q) for p, q in zip(y, want[1]))


def test_replayed_capture():
    """A captured call replayed on new logits, targets and advantages between eager
    calls: the eager bits each time."""
    z, tg, cu, cud, old, adv, ref = _policy_inputs([80, 60], 32003, B, 16)
    run = lambda: (*ops.policy_loss(z, tg, cu, old, adv, ref, kl_coef=0.05, cu_device=cud),  # noqa: E731
                   *ops.preference_loss(z, tg, cu, beta=0.01, cu_device=cud),
                   ops.token_logprobs(z, tg), ops.token_logprobs_backward(z, tg, adv))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k in range(4):
        new = _policy_inputs([80, 60], 32003, B, 20 + 2 * k)
        for t, n in zip((z, tg, old, adv, ref), (new[0], new[1], new[4], new[5], new[6])):
            t.copy_(n)
        want = run()
        for t in got:
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k


def test_offsets_beyond_32_bits():
    """Rows past element 2^31 of the logits, read and written; rows that do not count
    are written (zeros) and not read."""
    V, T = 128256, 16800
    z = torch.empty((T, V), dtype=B, device="cuda").fill_(float("nan"))
    tg = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    tail, tt, _ = make([3], V, B, 40, counted=1.0)
    z[-3:] = tail
    tg[-3:] = tt
    assert z.numel() > 1 << 31
    r = Rows(tail, tt)
    check(ops.token_logprobs(z, tg)[-3:], r.lp, r.E * U + U * r.lp.abs(), "logps")
    c = torch.ones(T, device="cuda")
    g = ops.token_logprobs_backward(z, tg, c, dlogits=z)
    one = torch.ones(3, dtype=torch.float64, device="cuda")
    check(g[-3:], r.grad(one), r.grad_bound(one, 0 * one, HALF[B]), "dlogits")
    assert not g[:-3].any()
