"""Drawing tokens from logits, on the GPU against float64 (NumPy).

A token is a whole number: it has to be the reference's.  The kernel's weights are
float64 and its sums whole numbers of 2^-38 or less of the largest weight; a border of
the inputs below comes closer than that to a row's number once in some 10^8 rows.  A
logarithm is rounded to float32 once."""
import math

import numpy as np
import pytest
import torch

import paper_2608_19889_amd as ops

pytestmark = pytest.mark.gpu
F, B = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def reference(z, u, t=1.0, k=0, p=1.0, low=0.0):
    """One row: (token, log-probability)."""
    z, t, p, low, u = z.astype(np.float64), *(np.float64(np.float32(x)) for x in (t, p, low, u))
    z = np.where(np.isnan(z), -INF, z)
    top = z.max()
    if top == -INF:
        return -1, 0.0
    if not t > 0:
        return int(np.argmax(z)), 0.0
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        w = np.where(z == top, 1.0, np.where(z == -INF, 0.0, np.exp((z - top) / t)))
        w = np.where(np.isnan(w), 0.0, w)
    down = np.argsort(-z, kind="stable")
    if 0 < k < len(z):
        w[down[k:]] = 0
    if p < 1:
        sums = np.cumsum(w[down])
        n = int(np.searchsorted(sums, max(p, 0) * sums[-1], side="left")) + 1
        w[down[n:]] = 0
    if low > 0:
        w[w < min(low, 1)] = 0
    sums = np.cumsum(w)
    u = 0.0 if math.isnan(u) else min(max(u, 0.0), 1.0)
    i = int(np.searchsorted(sums, u * sums[-1], side="right"))
    i = min(i, int(np.flatnonzero(w)[-1]))
    return i, math.log(w[i]) - math.log(sums[-1])


def check(z, u, **kw):
    """kw: numbers, or tensors over the rows"""
    tokens, logps = ops.sample_tokens(z, u, **kw)
    assert tokens.dtype == torch.int32 and logps.dtype == F
    of = lambda name, r, other: kw[name][r].item() if isinstance(kw.get(name), torch.Tensor) else kw.get(name, other)  # noqa: E731
    zs, us = z.float().cpu().numpy(), u.cpu().numpy()
    for r in range(len(zs)):
        token, lp = reference(zs[r], us[r], of("temperature", r, 1.0), of("top_k", r, 0), of("top_p", r, 1.0),
                              of("min_p", r, 0.0))
        assert int(tokens[r]) == token, (r, int(tokens[r]), token)
        assert abs(float(logps[r]) - lp) <= 2.0 ** -24 * abs(lp) + 1e-9, (r, float(logps[r]), lp)
    return tokens, logps


def logits(rows, V, dtype=F, seed=0, ld=None, peak=10.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((rows, ld or V), NAN, device="cuda", dtype=dtype)
    z = 2 * torch.randn((rows, V), generator=g, device="cuda")
    n = min(V, 40)
    z[:, torch.randperm(V, generator=g, device="cuda")[:n]] += peak * torch.rand((rows, n), generator=g, device="cuda")
    wide[:, :V] = z
    return wide[:, :V], torch.rand((rows,), generator=g, device="cuda")


FILTERS = {"whole": {}, "k": dict(top_k=17), "p": dict(top_p=0.9), "min": dict(min_p=0.02), "cold": dict(temperature=0.3),
           "hot": dict(temperature=3.0, top_p=0.99), "all": dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.01),
           "greedy": dict(temperature=0.0, top_k=5, top_p=0.3), "k+p": dict(top_k=300, top_p=0.8),
           "most": dict(top_k=1 << 30, top_p=0.9999)}


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 1000, 2048, 2049, 32000, 50257, 128256])
@pytest.mark.parametrize("kw", FILTERS.values(), ids=FILTERS.keys())
def test_sizes_and_filters(kw, V, dtype):
    z, u = logits(7, V, dtype, seed=V)
    check(z, u, **kw)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("kw", FILTERS.values(), ids=FILTERS.keys())
def test_flat_rows(kw, dtype):
    """Nothing stands out: a filter's border is among most of the vocabulary."""
    z, u = logits(5, 40000, dtype, seed=4, peak=0.0)
    check(0.3 * z, u, **kw)


@pytest.mark.parametrize("kw", FILTERS.values(), ids=FILTERS.keys())
@pytest.mark.parametrize("V,dtype", [(262144, F), (262145, F), (300001, B), (1 << 22, F)])
def test_largest_vocabularies(V, dtype, kw):
    check(*logits(2, V, dtype, seed=V % 1000), **kw)
    check(*logits(2, V, dtype, seed=V % 1000, peak=0.0), **kw)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("V,ld", [(999, 1003), (50257, 50272), (4096, 4097)])
def test_strides(V, ld, dtype):
    z, u = logits(9, V, dtype, ld=ld)
    for kw in ({}, FILTERS["all"]):
        check(z, u, **kw)
    wide = torch.randn((4, V + 9), device="cuda").to(dtype)
    check(wide[:, 3:3 + V], u[:4], **FILTERS["p"])


@pytest.mark.parametrize("V", [10, 1000, 70000])
def test_equal_logits(V):
    """Of equal logits the lower indices are kept; whole numbers of equal weights decide
    exactly."""
    z = torch.full((8, V), 1.5, device="cuda")
    u = torch.tensor([0.0, 0.1, 0.25, 0.5, 0.75, 0.99, 0.9999999, 0.3], device="cuda")
    for kw in ({}, dict(top_k=3), dict(top_p=0.5), dict(top_k=V // 2, top_p=0.5), dict(min_p=1.0), dict(top_p=0.3)):
        tokens, logps = ops.sample_tokens(z, u, **kw)
        n = kw.get("top_k", V)
        if "top_p" in kw:
            n = math.ceil(float(np.float32(kw["top_p"])) * n)
        want = [min(int(float(x) * n), n - 1) for x in u.cpu()]
        assert tokens.tolist() == want, kw
        assert np.allclose(logps.cpu().numpy(), -math.log(n), atol=1e-6)
    z[:, V // 2] = 2.0  # one above the others
    z[:, 1] = -1.0
    for kw in (dict(top_k=3), dict(top_k=4, temperature=0.5), dict(top_p=0.4, top_k=5)):
        check(z, u, **kw)


def test_numbers_outside_the_unit_interval():
    z, _ = logits(7, 3001)
    u = torch.tensor([-1.0, 0.0, 1.0, 2.0, NAN, -INF, INF], device="cuda")
    for kw in ({}, dict(top_k=5), dict(top_p=0.5)):
        check(z, u, **kw)


@pytest.mark.parametrize("dtype", [F, B])
def test_infinities_and_nan(dtype):
    z, u = logits(9, 5000, dtype)
    z[0] = -INF
    z[1] = NAN
    z[2, 1:] = -INF
    z[3, :4990] = -INF
    z[4, ::3] = NAN
    z[5, 7], z[5, 4000], z[5, 4500] = INF, INF, INF
    z[6] = INF
    z[7, 4999] = NAN
    z[8, ::2] = -INF
    for kw in FILTERS.values():
        t, lp = check(z, u, **kw)
        assert t[:2].tolist() == [-1, -1] and lp[:2].tolist() == [0, 0]
    # extreme values and both zeros
    z = torch.tensor([[3e38, -3e38, 0.0, -0.0], [0.0, -0.0, 0.0, -1e-45], [-3e38, -3e38, -INF, -3.1e38]], device="cuda").to(dtype)
    for uu in (0.0, 0.3, 0.6, 0.99):
        for kw in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=1e-6), dict(temperature=INF),
                   dict(temperature=1e30)):
            check(z, torch.full((3,), uu, device="cuda"), **kw)


def test_settings_of_each_row():
    z, u = logits(64, 20011, seed=9)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda: torch.rand((64,), generator=g, device="cuda")  # noqa: E731
    kw = dict(temperature=r() * 2, top_k=(r() * 100).int(), top_p=0.5 + 0.5 * r(), min_p=0.1 * r())
    for name, odd in (("temperature", [0.0, -1.0, NAN, INF, 1e-30]), ("top_p", [1.0, 2.0, 0.0, -3.0, NAN, INF, 1e-9]),
                      ("min_p", [0.0, -1.0, 2.0, NAN, INF, 1.0]), ("top_k", [0, -5, 20011, 20010, 2147483647, 1])):
        kw[name][7:7 + len(odd)] = torch.tensor(odd, dtype=kw[name].dtype, device="cuda")
        kw[name][40:40 + len(odd)] = torch.tensor(odd, dtype=kw[name].dtype, device="cuda")
    check(z, u, **kw)
    check(z, u, temperature=kw["temperature"], top_p=0.9)
    check(z, u, top_k=kw["top_k"], temperature=0.6)


def test_shares_of_many_draws():
    """The numbers (i + 1/2) / n give every token as often as its weight says."""
    n = 4096
    z = torch.tensor([2.0, 0.0, -1.0, 1.0, 3.0, -INF, 2.5], device="cuda").repeat(n, 1)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    t, lp = ops.sample_tokens(z, u, temperature=0.9)
    w = torch.softmax(z[0].double() / float(np.float32(0.9)), 0).cpu()
    count = torch.bincount(t.long().cpu(), minlength=7)
    assert (count - n * w).abs().max() <= 1
    assert torch.allclose(lp.cpu().double(), torch.log(w[t.long().cpu()]), atol=1e-6)


def test_many_rows_and_none():
    z, u = logits(3000, 257, seed=2)
    check(z, u, top_p=0.9)
    t, lp = ops.sample_tokens(z[:0], u[:0])
    assert t.shape == (0,) and lp.shape == (0,)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("kw", FILTERS.values(), ids=FILTERS.keys())
def test_more_rows_than_compute_units(kw, dtype):
    """More than 256 rows take smaller workgroups: few candidates, many, and equal ones."""
    check(*logits(300, 4099, dtype, seed=9), **kw)
    check(*logits(259, 20000, dtype, seed=10, peak=0.0), **kw)
    z, u = logits(257, 3000, dtype, seed=11)
    z = torch.where(z > 0, 1.5, z).to(dtype)
    check(z, u, **kw)


@pytest.mark.parametrize("V", [5000, 300001, 1 << 22])
def test_a_row_alone_and_among_many(V):
    """Larger and smaller workgroups give a row the same bits."""
    z = logits(3, V, B, seed=12)[0].repeat(100, 1)
    u = torch.rand((300,), generator=torch.Generator().manual_seed(13)).cuda()
    for kw in FILTERS.values():
        many, few = ops.sample_tokens(z, u, **kw), ops.sample_tokens(z[150:190], u[150:190], **kw)
        assert all(torch.equal(m[150:190], f) for m, f in zip(many, few)), kw


def test_out_stream_and_graph():
    z, u = logits(16, 32000)
    want, wlp = check(z, u, **FILTERS["all"])
    out = torch.full((16,), 5, dtype=torch.int32, device="cuda")
    got, _ = ops.sample_tokens(z, u, out=out, **FILTERS["all"])
    assert got is out and torch.equal(out, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, lp = ops.sample_tokens(z, u, stream=s, **FILTERS["all"])
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(lp, wlp)
    t = torch.full((16,), 0.8, device="cuda")
    k = torch.full((16,), 40, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gt, glp = ops.sample_tokens(z, u, temperature=t, top_k=k, top_p=0.95)
        gt2, glp2 = ops.sample_tokens(z, u)
    for i in range(4):
        z.copy_(logits(16, 32000, seed=i + 5)[0])
        u.copy_(torch.rand_like(u))
        t.fill_(0.5 + 0.2 * i)
        k.fill_(3 + 50 * i)
        graph.replay()
        et, elp = check(z, u, temperature=t, top_k=k, top_p=0.95)
        et2, elp2 = check(z, u)
        assert torch.equal(gt, et) and torch.equal(glp, elp) and torch.equal(gt2, et2) and torch.equal(glp2, elp2)


def test_inputs_are_left_as_they_were():
    z, u = logits(5, 1000, ld=1010)
    kept = z.clone()
    ops.sample_tokens(z, u, **FILTERS["all"])
    assert torch.equal(z, kept)
