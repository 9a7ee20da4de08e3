"""Rotating and appending to a paged cache, and attention over it with shared
prefixes, on the GPU against float64."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2608_19889_amd as ops
from paged_util import B, F, HALF, U, Paged, check

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rope_append

def rotated(x, pos, inv_freq, rot, interleaved, scale):
    """(float64 result, |x| + |y| of each pair)"""
    x = x.cpu().double()
    size = x.abs()
    out = x.clone()
    if rot:
        a = pos.double()[:, None, None] * inv_freq.cpu()
        c, s = torch.cos(a) * scale, torch.sin(a) * scale
        i = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
        j = i + 1 if interleaved else i + rot // 2
        out[..., i] = x[..., i] * c - x[..., j] * s
        out[..., j] = x[..., j] * c + x[..., i] * s
        size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return out, size


def check_append(p, rot, interleaved=False, scale=1.0, offsets=None, theta=10000.0, inplace=False, fused=False,
                 pad_rows=0, no_q=False):
    """A cosine or sine is off by 7 u: its argument's rounding (pi u / 2 of a half turn),
    the function's 4 ulp and the product with scale; the two products and their sum add
    2 u of (|x| + |y|) scale each at most: 10 u in all, and the stored value's rounding."""
    inv = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None
    q, k, v = p.q, p.k, p.v
    if fused:
        rows = torch.cat([q, k, v], 1)
        q, k, v = rows[:, :p.heads], rows[:, p.heads:p.heads + p.kv], rows[:, p.heads + p.kv:]
    if pad_rows:
        more = lambda t: torch.cat([t, torch.full_like(t[:1], float("nan")).expand(pad_rows, -1, -1)])  # noqa: E731
        q, k, v = more(q), more(k), more(v)
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    kc, vc = p.k_cache.cpu().double(), p.v_cache.cpu().double()
    kc_bound, vc_bound = torch.zeros_like(kc), torch.zeros_like(vc)
    seq = torch.repeat_interleave(torch.arange(len(p.new)), torch.tensor(p.new))
    slot = torch.tensor([int(p.lens[b]) + i for b, n in enumerate(p.new) for i in range(n)], dtype=torch.int64)
    pos = slot + (0 if offsets is None else torch.tensor(offsets)[seq])
    qr, qs = rotated(p.q, pos, inv, rot, interleaved, scale)
    kr, ks = rotated(p.k, pos, inv, rot, interleaved, scale)
    half = HALF[p.dtype]
    # dimensions behind the rotated ones are copied
    err = lambda r, s: torch.where(torch.arange(p.hd) < rot, 10 * U * s * abs(scale) * (1 + half) + half * r.abs(), 0.0)  # noqa: E731
    table = p.table.cpu()
    active = [int(p.lens[b]) >= 0 for b in seq.tolist()]
    for t in range(p.T):
        if not active[t]:
            continue
        col = int(slot[t]) // p.page
        page = int(table[seq[t], col]) if col < table.shape[1] else -1
        if 0 <= page < p.num_pages:
            at = (page, slice(None), int(slot[t]) % p.page)
            kc[at], kc_bound[at], vc[at] = kr[t], err(kr[t], ks[t]), p.v[t].cpu().double()
    before = torch.full((p.T + pad_rows, p.heads, p.hd), 7.0, dtype=p.dtype, device="cuda")
    out = q if inplace else before
    cu = p.cu_seqlens if not pad_rows else p.cu
    got = ops.rope_append(None if no_q else q, k, v, p.k_cache, p.v_cache, p.table, p.lens, inv, cu_seqlens=cu,
                          offsets=off, interleaved=interleaved, scale=scale, out=None if no_q else out)
    torch.cuda.synchronize()
    if no_q:
        assert got is None
    else:
        assert got is out
        keep = torch.tensor(active)
        check(got[:p.T][keep.cuda()], qr[keep], err(qr, qs)[keep], "q")
        if not inplace:
            assert (got[:p.T][~keep.cuda()] == 7).all() and (got[p.T:] == 7).all()
    nan = torch.isnan(kc)
    assert torch.equal(torch.isnan(p.k_cache.cpu()), nan)
    check(torch.nan_to_num(p.k_cache.cpu().double()), torch.nan_to_num(kc), kc_bound, "k cache")
    check(p.v_cache, vc, vc_bound, "v cache")


ONE = [(0, [(p, 1) for p in (0, 15, 16, 31, 40, 7)])]
RAGGED = [(0, [(0, 5), (15, 1), (16, 33), (3, 16), (0, 1), (47, 70)])]


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,hd,rot", [(9, 3, 64, 64), (4, 4, 128, 128), (28, 4, 128, 64), (2, 1, 64, 2),
                                             (3, 1, 64, 20), (5, 5, 128, 36), (25, 25, 64, 0)])
@pytest.mark.parametrize("groups", [ONE, RAGGED], ids=["one", "ragged"])
def test_append(groups, heads, kv, hd, rot, interleaved, dtype):
    check_append(Paged(groups, heads, kv, hd, dtype, seed=rot), rot, interleaved)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("page", [16, 48, 256])
def test_append_far_positions_pages_and_scale(page, dtype):
    p = Paged(RAGGED, 8, 2, 64, dtype, page=page)
    check_append(p, 64, scale=1.3, offsets=[0, 1 << 20, 2000000000, 999999, 2147483647, 5], theta=500000.0, fused=True)


@pytest.mark.parametrize("rot", [2, 64])
def test_append_reduces_far_angles(rot):
    """Far positions that are close to whole turns (numerators of 2 pi's continued fraction, and
    their neighbours): the small angle that is left has all its digits.  The bound is that of
    check_append, of the cosine and the sine each by itself (one of the two products is 0)."""
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    near = [710, 103993, 312689, 4272943, 10838702, 80143857, 411557987, 2137933792, 2147483647]
    near = near + [n - 1 for n in near] + [3 * 411557987, 26 * 80143857]
    left = []
    for n in near:
        turns = Fraction(n) / (2 * pi)
        left.append(float((turns - round(turns)) * 2 * pi))
    n = len(near)
    k = torch.zeros((n, 1, 64), device="cuda")
    k[..., :rot // 2] = 1
    kc, vc = (torch.zeros((n, 1, 16, 64), device="cuda") for _ in range(2))
    table, lens = torch.arange(n, dtype=torch.int32, device="cuda")[:, None], torch.zeros(n, dtype=torch.int32, device="cuda")
    inv = torch.ones(rot // 2, dtype=torch.float64, device="cuda")
    ops.rope_append(None, k, k, kc, vc, table, lens, inv, offsets=torch.tensor(near, dtype=torch.int32, device="cuda"))
    left = torch.tensor(left, dtype=torch.float64)[:, None].expand(-1, rot // 2)
    for i, f in ((0, torch.cos), (rot // 2, torch.sin)):
        want = f(left)
        check(kc[:, 0, 0, i:i + rot // 2], want, 11 * U * want.abs(), f.__name__)


def test_append_strides_in_place_and_without_queries():
    for kw in (dict(fused=True), dict(inplace=True), dict(fused=True, inplace=True), dict(no_q=True)):
        check_append(Paged(RAGGED, 6, 2, 64, B, seed=3), 64, **kw)
    # rows at odd elements: nothing is aligned to more than an element
    for dtype in (F, B):
        p = Paged(RAGGED, 6, 2, 64, dtype, seed=3)
        odd = torch.zeros((p.T, 6 * 64 + 3), dtype=dtype, device="cuda")
        view = odd.as_strided((p.T, 6, 64), (6 * 64 + 3, 64, 1), 1)
        view.copy_(p.q)
        p.q = view
        check_append(p, 64, inplace=True)
        assert (odd[:, 0] == 0).all() and (odd[:, -2:] == 0).all()


def test_append_leaves_what_is_behind_the_last_sequence_and_inactive_ones():
    p = Paged(RAGGED, 4, 2, 64, B)
    check_append(p, 64, pad_rows=3)
    p = Paged(ONE, 4, 2, 64, F)
    p.lens[1] = -1
    p.lens[4] = -2147483648
    check_append(p, 64)
    p = Paged(RAGGED, 4, 2, 64, F)
    p.lens[2] = -1
    check_append(p, 32)


def test_append_without_a_page_stores_nothing():
    p = Paged(RAGGED, 4, 2, 64, B, spare=4)
    p.table[2, 2], p.table[5, 3], p.table[5, 6], p.table[0, 0] = -1, p.num_pages, 2147483647, -2147483648
    check_append(p, 64)
    p = Paged(ONE, 4, 2, 64, F)
    p.lens[0], p.lens[3] = 1 << 30, p.table.shape[1] * p.page  # past the row
    check_append(p, 64, offsets=[0] * 6)


def test_append_offsets_past_32_bits():
    """An element of the cache past 2^31 elements (4 GiB of bf16)."""
    pages, page, kv, hd = (1 << 31) // (16 * 2 * 128) + 8, 16, 2, 128
    k_cache, v_cache = (torch.zeros((pages, kv, page, hd), dtype=B, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1], [3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([9, 2], dtype=torch.int32, device="cuda")
    k, v, q = (torch.randn(2, n, hd, device="cuda").to(B) for n in (kv, kv, 4))
    ops.rope_append(None, k, v, k_cache, v_cache, table, lens)
    assert torch.equal(k_cache[pages - 1, :, 9], k[0]) and torch.equal(v_cache[pages - 1, :, 9], v[0])
    assert torch.equal(k_cache[3, :, 2], k[1])
    k_cache[pages - 1, :, 9] = 0
    assert int(k_cache[pages - 1].count_nonzero()) == 0
    lens[0] = 0
    k_cache[pages - 1, :, 0], v_cache[pages - 1, :, 0] = k[0], v[0]
    out = ops.prefix_attention(q, k_cache, v_cache, table, lens)
    assert torch.equal(out[0], v[0].repeat_interleave(2, 0))


# ------------------------------------------------------------------ prefix_attention

def check_attention(p, scale=None):
    ref = p.attention(scale=scale)
    got, lse = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, scale=scale, want_lse=True,
                                    **p.attention_args())
    torch.cuda.synchronize()
    check(got, ref[0], ref[1], "out")
    check(lse, ref[2], ref[3], "lse")


HEADS = [(9, 3, 64), (28, 4, 128), (32, 8, 64), (4, 4, 128), (7, 1, 64), (25, 25, 64), (40, 1, 128)]
DECODE = {
    "one": [(1, [(0, 1)])],
    "tail": [(63, [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1)]), (64, [(62, 1), (63, 1), (64, 1)]), (65, [(127, 1)])],
    "no prefix": [(0, [(0, 1), (100, 1)]), (0, [(17, 1)])],
    "groups": [(200, [(5, 1)] * 3), (1, [(300, 1)]), (129, [(0, 1), (33, 1), (7, 1), (64, 1), (9, 1)])],
    "many": [(150, [(i % 23, 1) for i in range(40)])],
}
CHUNKS = {
    "chunk": [(70, [(0, 5), (15, 1), (40, 33)])],
    "long chunk": [(0, [(0, 130)]), (33, [(3, 70), (64, 64), (0, 1)])],
    "empty chunks": [(20, [(0, 0), (5, 3), (8, 0)]), (9, [(0, 2)])],
}


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("heads,kv,hd", HEADS)
@pytest.mark.parametrize("groups", DECODE.values(), ids=DECODE.keys())
def test_attention_of_single_tokens(groups, heads, kv, hd, dtype):
    check_attention(Paged(groups, heads, kv, hd, dtype))


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("heads,kv,hd", HEADS[:5])
@pytest.mark.parametrize("groups", CHUNKS.values(), ids=CHUNKS.keys())
def test_attention_of_chunks(groups, heads, kv, hd, dtype):
    check_attention(Paged(groups, heads, kv, hd, dtype, seed=1))


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("page", [32, 48, 256])
def test_attention_pages_that_end_inside_a_tile(page, dtype):
    check_attention(Paged(DECODE["tail"] + CHUNKS["chunk"], 8, 2, 128, dtype, page=page))


@pytest.mark.parametrize("dtype", [F, B])
def test_attention_long_prefix_in_many_parts(dtype):
    check_attention(Paged([(5000, [(700, 1), (3, 1)]), (1, [(2500, 1)])], 4, 1, 64, dtype))
    check_attention(Paged([(3001, [(0, 40), (90, 1)])], 8, 1, 128, dtype))


@pytest.mark.parametrize("dtype", [F, B])
def test_attention_masked_rows_and_places(dtype):
    # inactive sequences, prefixes of no keys, missing pages, lengths past the table
    p = Paged(DECODE["groups"], 8, 2, 64, dtype)
    p.lens[1] = -1
    p.lens[8] = -5
    p.prefix_lens[2] = -3
    check_attention(p)
    p = Paged(CHUNKS["chunk"], 8, 2, 64, dtype)
    p.table[2, 1] = -1
    p.prefix_table[0, 0], p.prefix_table[0, 3] = p.num_pages, -2147483648
    check_attention(p)
    p = Paged(DECODE["one"], 8, 2, 64, dtype)
    p.table[0, 0] = -7
    p.prefix_table[0, 0] = 1 << 30
    check_attention(p)  # a row without a key
    assert float(ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens).abs().max()) == 0
    p = Paged(DECODE["tail"], 8, 2, 64, dtype, junk=False)
    p.prefix_lens[0], p.lens[2] = p.prefix_table.shape[1] * 16, p.table.shape[1] * 16 - 1
    want = p.attention()
    p.prefix_lens[0], p.lens[2] = 1 << 30, 2147483647
    got = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args())
    check(got, want[0], want[1], "lengths past the table")


@pytest.mark.parametrize("dtype", [F, B])
def test_attention_later_tokens_do_not_show(dtype):
    """NaN and infinities in a chunk's later tokens leave the earlier ones as they are."""
    p = Paged([(40, [(20, 12), (0, 70)])], 4, 2, 64, dtype)
    want = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args()).clone()
    for b, j, val in ((0, 25, math.nan), (0, 27, math.inf), (0, 28, -math.inf), (1, 33, math.inf), (1, 64, math.nan)):
        page, at = int(p.table[b, j // 16]), j % 16
        p.k_cache[page, :, at, ::3] = val
        p.v_cache[page, :, at, ::2] = val
    got = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args())
    assert torch.equal(got[:5], want[:5]) and torch.equal(got[12:12 + 33], want[12:12 + 33])
    # an infinite value that is attended to shows, at its dimensions only
    p = Paged([(40, [(20, 12)])], 4, 2, 64, dtype)
    p.v_cache[int(p.table[0, 1]), :, 25 - 16, 3] = math.inf
    p.v_cache[int(p.table[0, 1]), :, 27 - 16, 3] = -math.inf
    got = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args())
    assert torch.isfinite(got[:5]).all() and (got[5:7, :, 3] == math.inf).all() and torch.isnan(got[7:, :, 3]).all()
    assert torch.isfinite(got[..., :3]).all() and torch.isfinite(got[..., 4:]).all()


@pytest.mark.parametrize("dtype", [F, B])
def test_attention_scores_far_apart(dtype):
    """One key takes all the weight, wherever it stands; scores that grow along the keys
    rescale what was summed before."""
    p = Paged([(300, [(150, 1), (0, 1)])], 4, 2, 64, dtype)
    p.q *= 12
    check_attention(p)
    check_attention(p, scale=0.0)
    check_attention(p, scale=1e-42)
    check_attention(p, scale=-0.7)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_many_rows_with_scores_far_apart(hd, dtype):
    """More than 128 rows of one key head, whose scores grow inside a tile of keys."""
    p = Paged([(600, [(5 * i % 50, 1) for i in range(20)])], 8, 1, hd, dtype)
    p.q *= 12
    check_attention(p)
    p = Paged([(70, [(3, 50), (0, 1)])], 12, 2, hd, dtype)
    p.q *= 12
    check_attention(p)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("spread", [1, 12])
@pytest.mark.parametrize("seqs,heads,hd", [(75, 16, 64), (18, 32, 128)])
def test_attention_many_tiles_in_a_row(seqs, heads, hd, spread, dtype):
    """A prefix so long that every workgroup goes through many tiles of keys."""
    N, kv = 50011, 4
    p = Paged([(N, [(0, 1)] * seqs)], heads, kv, hd, dtype, junk=False)
    p.q *= spread
    G, q = heads // kv, p.q.cpu().double()
    prefix, own = p.prefix_table[0].cpu().long(), p.table[:, 0].cpu().long()
    got, lse = (t.cpu().double() for t in ops.prefix_attention(
        p.q, p.k_cache, p.v_cache, p.table, p.lens, want_lse=True, **p.attention_args()))
    kc, vc = p.k_cache.cpu(), p.v_cache.cpu()
    for h in range(kv):
        k, v = (c[prefix, h].reshape(-1, hd)[:N].double() for c in (kc, vc))
        k1, v1 = (c[own, h, 0].double().repeat_interleave(G, 0) for c in (kc, vc))
        rows = q[:, h * G:(h + 1) * G].reshape(-1, hd)
        s = torch.cat([rows @ k.T, (rows * k1).sum(1, keepdim=True)], 1) * hd ** -0.5
        # the bound of Paged.attention
        d = (hd + 2) * U * torch.maximum((rows.abs() @ k.abs().T).amax(1), (rows * k1).abs().sum(1)) * hd ** -0.5
        x = s.amax(1, keepdim=True) - s
        w = torch.softmax(s, 1)
        eps = (2 * d + (w * (3 * x + 8)).amax(1) * U + (8 + N + 1) * U)[:, None]
        out, size = w[:, :N] @ v + w[:, N:] * v1, w[:, :N] @ v.abs() + w[:, N:] * v1.abs()
        bound = (2 * eps + (HALF[B] if dtype == B else 0)) * size
        at = (slice(None), slice(h * G, (h + 1) * G))
        check(got[at].reshape(-1, hd), out, bound + HALF[dtype] * (out.abs() + bound), ("out", h))
        total = torch.logsumexp(s, 1)
        check(lse[at].reshape(-1), total, eps[:, 0] + 4 * U * (1 + total.abs() + s.abs().amax(1)), ("lse", h))


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("size", [2e36, 2.0 ** -122])
@pytest.mark.parametrize("growth", [7.9, 0.0])
@pytest.mark.parametrize("groups,heads,kv,hd", [
    ([(150, [(20, 1)] * 5)], 8, 2, 64),           # 20 rows
    ([(150, [(3, 1)] * 40)], 8, 1, 128),          # 320
    ([(0, [(99, 1), (140, 1)])], 8, 2, 128),      # 4, a wavefront's
    ([(0, [(99, 1), (140, 1)])], 8, 2, 64),
    ([(70, [(90, 60), (5, 1)])], 4, 2, 64),       # many new tokens
])
def test_attention_values_near_the_ends_of_the_range(groups, heads, kv, hd, growth, size, dtype):
    """Large and small finite values, and scores that grow along the keys by less than 8 (in
    base 2) or not at all: sums of weights and values stay in range where weights of 1 at most
    do."""
    p = Paged(groups, heads, kv, hd, dtype)
    p.q.zero_()
    p.q[..., 0] = 1
    for table, lens in ((p.table, [a + b for a, b in zip(p.past, p.new)]), (p.prefix_table, p.prefix)):
        for row, n in zip(table.cpu().tolist(), lens):
            for j in range(n):
                at = (row[j // p.page], slice(None), j % p.page)
                p.k_cache[at] = 0
                p.k_cache[(*at, 0)] = growth * j / n
                p.v_cache[at] = size * (1 + torch.rand((kv, hd), generator=torch.Generator().manual_seed(j))).to(dtype).cuda()
    check_attention(p, scale=math.log(2))


@pytest.mark.parametrize("dtype", [F, B])
def test_attention_more_sequences_than_threads(dtype):
    """Several segments to a thread of the plan; groups of none, sequences that take no part."""
    g = torch.Generator().manual_seed(3)
    some = lambda n: torch.randint(0, n, (1,), generator=g).item()  # noqa: E731
    p = Paged([(some(40), [(some(20), 1)] * some(5)) for _ in range(330)] + [(9, [(3, 1)])], 2, 1, 64, dtype)
    assert len(p.past) + len(p.prefix) > 2 * 420
    p.lens[::7] = -1
    p.lens[40:300] = -1  # a long run of segments without work
    check_attention(p)
    p = Paged([(some(30), [(some(9), some(3))] * (1 + some(3))) for _ in range(280)], 20, 1, 64, dtype)
    assert len(p.past) + len(p.prefix) > 512
    p.lens[::5] = -9
    check_attention(p)


def test_attention_strides_and_in_place():
    for dtype in (F, B):
        p = Paged(CHUNKS["chunk"], 6, 2, 64, dtype)
        wide = torch.zeros((p.T, 6 * 64 + 5), dtype=dtype, device="cuda")
        view = wide.as_strided((p.T, 6, 64), (6 * 64 + 5, 64, 1), 3)
        view.copy_(p.q)
        p.q = view
        check_attention(p)
        ref = p.attention()
        got = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, out=p.q, **p.attention_args())
        assert got.data_ptr() == view.data_ptr()
        check(got, ref[0], ref[1], "in place")
        assert (wide.as_strided((p.T, 3), (6 * 64 + 5, 1), 0) == 0).all() and (wide[:, -2:] == 0).all()


def test_attention_rows_behind_the_last_sequence_are_left():
    p = Paged(CHUNKS["chunk"], 6, 2, 64, B)
    ref = p.attention()
    q = torch.cat([p.q, torch.full((3, 6, 64), float("nan"), dtype=B, device="cuda")])
    out = torch.full_like(q, 7)
    got = ops.prefix_attention(q, p.k_cache, p.v_cache, p.table, p.lens, out=out, **p.attention_args())
    check(got[:p.T], ref[0], ref[1], "out")
    assert (got[p.T:] == 7).all()


def test_attention_more_sequences_than_groups_cover():
    p = Paged(DECODE["groups"], 8, 2, 64, B)
    p.cu_groups = [0, 2, 3, 5]  # the last four have no prefix
    check_attention(p)


def test_more_tokens_than_a_grid_dimension_has_threads():
    """2^24 tokens and some, most of them of a sequence that takes no part."""
    n, hd = 1 << 24, 64
    cu = [0, 100, n, n + 70]
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.empty((n + 70, 1, hd), dtype=B, device="cuda")
    ends = torch.cat([torch.arange(100), n + torch.arange(70)]).cuda()
    q[ends] = torch.randn((170, 1, hd), generator=g, device="cuda").to(B)
    kc, vc = (torch.zeros((12, 1, 16, hd), dtype=B, device="cuda") for _ in range(2))
    table = torch.full((3, 7), -1, dtype=torch.int32)
    table[0], table[2, :5] = torch.arange(7), torch.arange(7, 12)
    table, lens = table.cuda(), torch.tensor([0, -1, 0], dtype=torch.int32).cuda()
    assert ops.rope_append(None, q, q, kc, vc, table, lens, cu_seqlens=cu) is None
    for c in (kc, vc):
        assert torch.equal(c[:7].view(112, hd)[:100], q[:100, 0]) and torch.equal(c[7:].view(80, hd)[:70], q[n:, 0])
    out = torch.full_like(q, 5)
    ops.prefix_attention(q, kc, vc, table, lens, cu_seqlens=cu, out=out)
    few = ops.prefix_attention(q[ends].contiguous(), kc, vc, table[::2].contiguous(), lens[::2].contiguous(),
                               cu_seqlens=[0, 100, 170])
    assert torch.equal(out[ends], few) and not out[100:n].any()


def test_as_many_sequences_as_are_taken_with_long_tables():
    """4096 tokens of 40 heads a kv head, tables of 2^18 keys that list few, against the same
    64 at a time.  Each is off by (2 eps + 2 u) max |v| at most, eps as in Paged.attention."""
    n, kv, G, hd, columns = 4096, 8, 40, 64, (1 << 18) // 16
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn((n, kv * G, hd), generator=g, device="cuda")
    kc, vc = (torch.randn((n + 9, kv, 16, hd), generator=g, device="cuda") for _ in range(2))
    lens = torch.randint(0, 16, (n,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((n, columns), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(9, n + 9, device="cuda")
    prefix = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    prefix[0, :9] = torch.arange(9, device="cuda")
    plens = torch.tensor([135], dtype=torch.int32, device="cuda")
    got = ops.prefix_attention(q, kc, vc, table, lens, prefix_table=prefix, prefix_lens=plens)
    keys = torch.cat([kc[:9].abs().amax((0, 2)), kc[9:].abs().amax((0, 2))]).amax(0)  # [hd]
    score = float((q.abs() * keys).sum(2).max()) * hd ** -0.5
    eps = 2 * (hd + 2) * U * score + (3 * 2 * score + 8) * U + (8 + 151) * U
    bound = 2 * (2 * eps + 2 * U) * float(vc.abs().max())
    for i in range(0, n, 64):
        part = slice(i, i + 64)
        want = ops.prefix_attention(q[part], kc, vc, table[part, :1].contiguous(), lens[part],
                                    prefix_table=prefix[:, :9].contiguous(), prefix_lens=plens)
        assert float((got[part] - want).abs().max()) <= bound, i


def test_same_bits_again():
    for dtype in (F, B):
        p = Paged([(2000, [(300, 1), (3, 1)]), (70, [(9, 20)])], 8, 2, 128, dtype)
        a, b = (ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args()) for _ in range(2))
        assert torch.equal(a, b)


# ------------------------------------------------------------------ streams and graphs

def test_other_stream():
    p = Paged(CHUNKS["chunk"], 8, 2, 64, B)
    want = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **p.attention_args())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, stream=s, **p.attention_args())
    s.synchronize()
    assert torch.equal(got, want)


def test_captured_decode_step_follows_its_lengths():
    """One graph of append and attention, replayed while lengths, tables and tokens
    change on the device, against eager calls."""
    p = Paged([(100, [(13, 1), (0, 1), (31, 1)]), (20, [(63, 1)])], 8, 2, 64, B)
    table = torch.full((4, 8), -1, dtype=torch.int32, device="cuda")
    table[:, :p.table.shape[1]] = p.table
    free = iter(sorted(set(range(p.num_pages + 20)) - set(p.table.flatten().tolist()) -
                       set(p.prefix_table.flatten().tolist())))
    grow = lambda c: torch.cat([c, torch.zeros((20, *c.shape[1:]), dtype=c.dtype, device="cuda")])  # noqa: E731
    kc, vc = grow(p.k_cache), grow(p.v_cache)
    kc2, vc2 = kc.clone(), vc.clone()
    groups = torch.tensor(p.cu_groups, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([100, 100, 100, 20], dtype=torch.int32, device="cuda")
    inv = 1e4 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device="cuda") / 64)
    lens = p.lens.clone()
    q, k, v = p.q.clone(), p.k.clone(), p.v.clone()

    def step(kc, vc):
        r = ops.rope_append(q, k, v, kc, vc, table, lens, inv, offsets=offsets)
        return ops.prefix_attention(r, kc, vc, table, lens, prefix_table=p.prefix_table, prefix_lens=p.prefix_lens,
                                    cu_groups=p.cu_groups, groups_device=groups, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(kc2, vc2)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(kc, vc)
    for i in range(5):
        for b in range(4):
            col = int(lens[b]) // 16
            if int(table[b, col]) < 0:
                table[b, col] = next(free)
        for t in (q, k, v):
            t.copy_(torch.randn_like(t, dtype=F))
        graph.replay()
        want, want_lse = step(kc2, vc2)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), i
        assert torch.equal(torch.nan_to_num(kc), torch.nan_to_num(kc2))
        lens += 1


def test_captured_call_of_one_group_without_its_sums():
    p = Paged([(70, [(13, 1), (0, 1), (31, 1)])], 8, 2, 64, B)
    kw = dict(prefix_table=p.prefix_table, prefix_lens=p.prefix_lens)
    step = lambda: ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, **kw)  # noqa: E731
    assert torch.equal(step(), ops.prefix_attention(p.q, p.k_cache, p.v_cache, p.table, p.lens, cu_groups=[0, 3], **kw))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        p.q.copy_(torch.randn_like(p.q, dtype=F))
        p.prefix_lens.fill_(70 - 9 * i)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_a_buffer_counts_as_modified():
    p = Paged(ONE, 4, 2, 64, F)
    versions = [t._version for t in (p.k_cache, p.v_cache, p.q)]
    ops.rope_append(p.q, p.k, p.v, p.k_cache, p.v_cache, p.table, p.lens, out=p.q)
    assert all(t._version > n for t, n in zip((p.k_cache, p.v_cache, p.q), versions))
