"""Layer norm on the GPU where a workgroup goes through several rows (the next row is
loaded while one is reduced, the slots of the row's sums alternate, the columns' sums
build up in registers), every row width, ragged last rounds, against float64.

u = 2^-24.  A thread holds at most 32 values of a row (4 groups of 8), so a row's sum is
8 + 4 + 6 lane steps + 4 wavefront steps additions deep, below the 64 of
test_gpu_layernorm, whose bounds of y and dx hold.  A column's sum takes as many
additions as a workgroup has rounds, 4 over its wavefronts, one for every 64th
workgroup, and 64: that many u of the sum of the absolute terms, beside the terms' own
errors.
"""
import pytest
import torch

import autograd_util as ag
import paper_2608_19889_amd as ops
from test_gpu_gpt2 import gpt2_shape
from test_gpu_layernorm import B, EPS, F, HALF, U, check, check_forward, rows, stats
from test_gpu_train_losses import check_all, setup

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("types", [(F, F, F), (B, B, B), (F, B, B)], ids=["f32", "bf16", "mixed"])
size = lambda s: "%dx%d" % s  # noqa: E731

# more rounds than one of each width's workgroups: (rows at once in a workgroup, most
# workgroups) forward 4 x 2048 up to 512 columns, 4 x 4096 to 1024, 4 x 512 to 2048, 16384
# above; backward 4 x 1024 to 1024 columns, 4 x 256 to 2048, 256 above
FORWARD = [(9001, 48), (24601, 509), (17001, 771), (33000, 1024), (6001, 1600), (2100, 2041), (16500, 2056),
           (32800, 2049), (16401, 4104), (16400, 8193), (16390, 16384)]
BACKWARD = [(9001, 48), (12301, 509), (9001, 771), (4500, 1024), (3333, 1600), (2100, 2041), (800, 2049), (803, 4096),
            (800, 8184), (515, 4097), (600, 16383), (770, 16384)]


@TYPES
@pytest.mark.parametrize("shape", FORWARD, ids=size)
def test_forward_of_several_rounds(shape, types):
    (r, c), (tx, ty, tp) = shape, types
    x = rows(r, c, tx, 1, pad=0 if c % 8 == 0 else 3, scale=2.0, offset=0.7)
    g, b = rows(1, c, tp, 3, scale=0.3, offset=1.0)[0], rows(1, c, tp, 4)[0]
    y = ops.layernorm(x, g, b, EPS, dtype=ty)
    for i in range(0, r, 4096):
        check_forward(x[i:i + 4096], g, b, y[i:i + 4096])
    if tx == ty:
        ops.layernorm(x, g, b, EPS, out=x)
        assert torch.equal(x, y)


def columns_bound(dy, d, r, top, n):
    """of dgain and dbias, for n additions in a row"""
    t = (dy * d * r).abs()
    return (n * U * t.sum(0) + 64 * U * (dy.abs() * (d.abs() + top) * r).sum(0) + 1e-45,
            n * U * dy.abs().sum(0) + 1e-45)


@TYPES
@pytest.mark.parametrize("shape", BACKWARD, ids=size)
def test_backward_of_several_rounds(shape, types):
    (R, C), (tx, ty, tp) = shape, types
    x = rows(R, C, tx, 5, pad=0 if C % 8 == 0 else 1, scale=2.0, offset=0.7)
    dy = rows(R, C, ty, 6)
    g = rows(1, C, tp, 7, scale=0.3, offset=1.0)[0]
    dx, dg, db = ops.layernorm_backward(dy, x, g, EPS)
    at_once, most = (4, 1024) if C <= 1024 else (4, 256) if C <= 2048 else (1, 256)
    turns = -(-R // at_once)
    rounds = -(-turns // most)
    assert rounds > 1
    d, r, top = stats(x)
    dyd, gd = dy.double(), g.double()
    k = dyd * gd
    big = lambda v: v.abs().amax(-1, keepdim=True)  # noqa: E731
    mean = lambda v: v.mean(-1, keepdim=True)  # noqa: E731
    want = r * (k - mean(k) - d * r * r * mean(k * d))
    check(dx, want, 64 * U * r * (big(k) + (big(d) + top) * r * r * mean((k * d).abs())
                                  + big(d) * r * r * top * mean(k.abs())) + (2 * U + HALF[dx.dtype]) * want.abs() + 1e-45)
    bg, bb = columns_bound(dyd, d, r, top, rounds + 4 + -(-turns // rounds) // 64 + 1 + 64)
    check(dg, (dyd * d * r).sum(0), bg)
    check(db, dyd.sum(0), bb)
    # the same bits in an input's buffer
    for over in ([x] if tx != ty else [x, dy]):
        keep = over.clone()
        got = ops.layernorm_backward(dy, x, g, EPS, dx=over)
        assert got[0] is over and all(torch.equal(p, q) for p, q in zip(got, (dx, dg, db)))
        over.copy_(keep)


# training steps of more rows than their 512 workgroups take at once: 4 each at a width of
# 512 or less, one above, of 256, 512 and 1024 threads
STEPS = {"hidden_64": (gpt2_shape(hidden=64, heads=1, layers=1, vocab=131, positions=800), [800, 777, 690]),
         "hidden_512": (gpt2_shape(layers=1, vocab=300, inter=512, positions=800), [733, 790, 640]),
         "hidden_640": (gpt2_shape(hidden=640, heads=10, layers=1, vocab=300, inter=640, positions=400), [310, 390, 3]),
         "hidden_2112": (gpt2_shape(hidden=2112, heads=33, layers=1, vocab=129, inter=64, positions=300), [300, 277]),
         "hidden_4160": (gpt2_shape(hidden=4160, heads=65, layers=1, vocab=65, inter=64, positions=300), [271, 260])}


@pytest.mark.parametrize("case", list(STEPS))
def test_training_step_of_several_rounds(case):
    shape, lens = STEPS[case]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 121)
    want, ref = ag.loss_and_grads(shape, w, seqs, ag.cross_entropy(tg))
    loss = m.loss_and_grads(flat, cu, targets, grads)
    assert abs(float(loss) - want) < 2e-3 * max(1.0, (shape["hidden_size"] / 896) ** 0.5)
    check_all(shape, seqs, grads, ref)
    m.close()
