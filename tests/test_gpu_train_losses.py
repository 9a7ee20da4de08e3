"""Training steps of the GPT-2 family and with the preference and policy losses,
against float64 automatic differentiation.

Bars per gradient tensor: those of test_gpu_train (same kernels and storage: bf16
between the kernels, float32 accumulation).  A loss's coefficients depend on the
model's own log-probabilities, which its bf16 storage moves by about 3e-3 a token
(the logits' bar of the parity tests): a ratio exp(l - old) or a margin of beta times
a sequence's sum moves its gradients by well under 1% of themselves, inside the
bars; ratios are kept 5% away from where they are clipped, where the gradient jumps.

The element-wise bar of the two losses' steps is wider.  Row r of a weight's gradient
is sum_t d_t[r] x_t over the tokens t, x_t the layer's normalized input.  In the mean
cross-entropy every token has the same weight; here a weight is -q A of either sign,
0 where clipped, and per sequence divided by its length, so one token of a short
sequence can carry a row alone.  That row's error is then that token's: e_t[r] x_t,
with |e_t| up to the 5e-2 of a token's own gradient (the bar of check_token_rows), and
its elements spread as x_t's, close to normal: the largest of n is sqrt(2 ln n) times
their root mean square.  So |g - r| <= 5e-2 sqrt(2 ln n) of the scale, 26% at n =
2^20.  (The storage alone, emulated in float64 by rounding what the kernels store to
bf16, gives 16.7% at a relative L2 error of 1.2e-2 in the last layer's q projection of
"llama" per sequence, one head's rows: dS = P (dP - D) cancels in the 5-token
sequence, and D comes from the stored bf16 output; measured 25% at 1.3e-2.)
"""
import math

import numpy as np
import pytest
import torch

import autograd_util as ag
import paper_2608_19889_amd as ops
from paper_2608_19889_amd import axon as ax
from parity_util import gpu_model, pack
from synthetic import model_weights, prompts, small_shape
from test_gpu_gpt2 import gpt2_shape
from test_gpu_train import ULP, _targets, check_gradient, check_token_rows

pytestmark = pytest.mark.gpu

GPT2 = {
    # one head, rows of 64 (a wavefront each in the layer norms' backward); one-token sequences
    "hidden_64": (gpt2_shape(hidden=64, heads=1, layers=2, vocab=131, positions=70), [33, 1, 64, 5]),
    "hidden_512": (gpt2_shape(layers=2, vocab=3000, positions=200), [37, 130, 65, 5]),
    "split_k": (gpt2_shape(layers=1, vocab=1001, positions=320), [200, 310, 90]),
    "xl_rows": (gpt2_shape(hidden=1600, heads=25, layers=1, vocab=500, inter=640, positions=64), [61, 30]),
    # layer norm rows of 512 and 1024 threads
    "hidden_2112": (gpt2_shape(hidden=2112, heads=33, layers=1, vocab=129, inter=64, positions=40), [33, 30]),
    "hidden_4160": (gpt2_shape(hidden=4160, heads=65, layers=1, vocab=65, inter=64, positions=40), [31, 1]),
}
FAMILIES = {"llama": (small_shape("1b", layers=2, vocab=1003, hidden=512, intermediate=1024), [37, 66, 65, 5]),
            "qwen": (small_shape("7b", layers=1, vocab=700, hidden=896, intermediate=320), [40, 33, 20, 71]),
            "gpt2": (gpt2_shape(layers=2, vocab=1003, positions=100), [37, 66, 65, 5])}


def setup(shape, lens, seed):
    w = model_weights(shape, seed=seed)
    ids = prompts(len(lens), max(lens), shape["vocab_size"], seed=seed + 1).numpy()
    seqs = [ids[i, :n] for i, n in enumerate(lens)]
    tg = np.concatenate(_targets(seqs, shape["vocab_size"], seed=seed + 2))
    m = gpu_model(shape, w, max_batch=len(lens), max_seq=max(lens))
    flat, cu = pack(seqs)
    grads = {k: torch.full(tuple(v.shape), float("nan"), dtype=torch.float32, device="cuda") for k, v in w.items()}
    return w, seqs, tg, m, flat, cu, torch.as_tensor(tg.astype(np.int32)).to("cuda"), grads


def check_weighted(name, g, r):
    """check_gradient with the element-wise bar of rows that one token may carry"""
    assert np.all(np.isfinite(g)), name
    scale = np.full(r.shape, float(np.sqrt(np.mean(r * r))))
    if r.ndim == 2:
        scale = np.maximum(scale, np.sqrt(np.mean(r * r, axis=1, keepdims=True)))
    err = np.abs(g - r)
    bar = max(32 * ULP, 5e-2 * math.sqrt(2 * math.log(r.size)))
    assert np.all(err <= bar * scale + 4 * ULP * np.abs(r)), (name, float((err / scale).max()), bar)
    rel = float(np.linalg.norm(g - r) / np.linalg.norm(r))
    assert rel < 3e-2, (name, rel)
    return rel, float((err / scale).max())


def check_all(shape, seqs, grads, ref, bars=check_gradient):
    for name, r in ref.items():
        rel, el = bars(name, grads[name].cpu().double().numpy(), r)
        print(f"  {name}: relative L2 {rel:.2e}, largest element error {el:.2e} x scale")
    emb = "transformer.wte.weight" if shape.get("model_type") == "gpt2" else "model.embed_tokens.weight"
    print("  token rows", check_token_rows(grads[emb].cpu().double().numpy(), ref[emb], np.concatenate(seqs)))


@pytest.mark.parametrize("case", list(GPT2))
def test_gpt2_loss_and_grads(case):
    shape, lens = GPT2[case]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 81)
    want, ref = ag.loss_and_grads(shape, w, seqs, ag.cross_entropy(tg))
    loss = m.loss_and_grads(flat, cu, targets, grads)
    print(case, float(loss), want)
    # the loss's bar grows with the root of the width, as test_gpu_train_tiles derives
    assert abs(float(loss) - want) < 2e-3 * max(1.0, (shape["hidden_size"] / 896) ** 0.5)
    check_all(shape, seqs, grads, ref)
    assert not grads["transformer.wpe.weight"][max(lens):].any()
    # a second call on another batch overwrites every gradient
    m.loss_and_grads(*pack(seqs[:1]), targets[:lens[0]], grads)
    _, ref = ag.loss_and_grads(shape, w, seqs[:1], ag.cross_entropy(tg[:lens[0]]))
    check_all(shape, seqs[:1], grads, ref)
    # and nothing is counted: zeros
    loss = m.loss_and_grads(flat, cu, torch.full_like(targets, -1), grads)
    assert float(loss) == 0 and all(not g.any() for g in grads.values())
    m.close()


@pytest.mark.parametrize("family", list(FAMILIES))
def test_preference_step(family):
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 84)
    lp, _ = ag.at_targets(torch.log_softmax(ag.logits(shape, {k: v.double() for k, v in w.items()}, seqs), -1), tg)
    sums = np.array([float(lp[a:b].sum()) for a, b in zip(cu, cu[1:])])
    ref_lp = sums + np.array([2.0, -3.0, -4.0, 1.0])
    want, ref = ag.loss_and_grads(shape, w, seqs, ag.preference(tg, cu, ref_lp, 0.1, 0.05))
    ref_d = torch.as_tensor(ref_lp, dtype=torch.float32, device="cuda")
    loss, seq, margins = m.preference_loss_and_grads(flat, cu, targets, grads, ref_d, beta=0.1, label_smoothing=0.05)
    # a token's log-probability is off by about 3e-3 (bf16 storage), a sum of n by up to
    # 6 sqrt(n) of that; the loss moves by at most beta times two such sums
    off = 6 * 3e-3 * np.sqrt(np.diff(cu))
    assert np.all(np.abs(seq.cpu().double().numpy() - sums) <= off)
    u = -0.1 * np.array([2.0 + 3.0, -4.0 - 1.0])
    pair = 0.1 * (off[0::2] + off[1::2])
    assert np.all(np.abs(margins.cpu().double().numpy() - u) <= pair)
    assert abs(float(loss) - want) <= pair.mean()
    check_all(shape, seqs, grads, ref, check_weighted)
    m.close()


def policy_inputs(shape, w, seqs, tg, seed):
    lp, ok = ag.at_targets(torch.log_softmax(ag.logits(shape, {k: v.double() for k, v in w.items()}, seqs), -1), tg)
    r = np.random.default_rng(seed)
    moved = 0.25 * r.standard_normal(len(tg))
    for edge in np.log([0.8, 1.3]):
        moved = np.where(np.abs(moved - edge) < 0.05, moved + 0.12, moved)
    old, ref = lp.numpy() - moved, lp.numpy() + 0.3 * r.standard_normal(len(tg))
    adv = r.standard_normal(len(tg)) + 0.4
    for v in (old, ref, adv):
        v[~ok.numpy()] = np.nan
    dev = [torch.as_tensor(v, dtype=torch.float32, device="cuda") for v in (old, adv, ref)]
    return lp, ok, old, adv, ref, dev


@pytest.mark.parametrize("per", [False, True])
@pytest.mark.parametrize("family", list(FAMILIES))
def test_policy_step(family, per):
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 87)
    lp, ok, old, adv, ref_lp, dev = policy_inputs(shape, w, seqs, tg, 90)
    want, ref = ag.loss_and_grads(shape, w, seqs, ag.policy(tg, cu, old, adv, ref_lp, 0.2, 0.3, 0.1, per))
    loss, stats, logps = m.policy_loss_and_grads(flat, cu, targets, grads, dev[0], dev[1], dev[2], clip_low=0.2,
                                                 clip_high=0.3, kl_coef=0.1, per_sequence=per)
    # each token's term moves by at most |A| q + k |e^g - 1| times 6 x 3e-3
    assert float((logps.cpu().double() - lp).abs().max()) <= 6 * 3e-3
    q = np.exp(np.where(ok, lp.numpy() - np.where(ok, old, 0), 0))
    assert abs(float(loss) - want) <= 6 * 3e-3 * float(np.nanmean(np.abs(adv) * np.minimum(q, 1.3)) + 0.1)
    check_all(shape, seqs, grads, ref, check_weighted)
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_scored_rollouts_then_a_policy_step(family):
    """The operators as they are used together: score the batch under the model
    (logits of every position, token_logprobs), give the result to policy_loss over
    those logits and to the model's own step; with old = the scored log-probabilities
    every ratio is 1 within the two passes' rounding, so nothing is clipped and the
    gradient is that of -A lp."""
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 93)
    logits, _ = m.prefill(flat, cu, all_logits=True)
    old = ops.token_logprobs(logits, targets)
    adv = torch.randn(len(tg), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) + 0.5
    loss, stats, logps, dlogits = ops.policy_loss(logits, targets, cu, old, adv, old, kl_coef=0.1)
    assert float(stats[1]) < 1e-9 and float(stats[2]) == 0
    same, sstats, slogps = m.policy_loss_and_grads(flat, cu, targets, grads, old, adv, old, kl_coef=0.1)
    assert float((slogps - old).abs().max()) <= 6 * 3e-3 * 2 and float(sstats[2]) == 0
    assert abs(float(same) - float(loss)) <= 6 * 3e-3 * 2 * float(adv.abs().max())
    a = adv.cpu().double()

    def plain(logp):
        lp, ok = ag.at_targets(logp, tg)
        return -(torch.where(ok, a, 0.0) * lp).sum() / ok.sum()
    _, ref = ag.loss_and_grads(shape, w, seqs, plain)
    check_all(shape, seqs, grads, ref, check_weighted)
    # the gradient at the logits, handed to a projection's backward by the caller, is the
    # one that token_logprobs_backward gives for the same coefficients
    n = int((targets >= 0).sum())
    same = ops.token_logprobs_backward(logits, targets, -adv / n)
    off = (same - dlogits).abs().max() / dlogits.abs().max()
    assert float(off) <= 2.0 ** -20
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_replayed_capture_of_a_step(family):
    """A captured policy step, replayed on other tokens and advantages between eager
    steps: the eager bits (the embedding's rows, sums of atomic additions, within
    their rounding)."""
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 96)
    other = {k: torch.empty_like(v) for k, v in grads.items()}
    old = torch.full((len(tg),), -6.5, device="cuda")
    adv = torch.randn(len(tg), device="cuda")
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    cuh = (ax.ctypes.c_int32 * len(cu))(*cu)
    out = torch.empty(2, 4 + len(tg), device="cuda")

    def step(g, o):
        arr, keep = ax.make_weights(g)
        at = o.data_ptr()
        ax._check(ax.lib().axon_policy_loss_and_grads(m._h, len(lens), flat.data_ptr(), cud.data_ptr(), cuh,
                                                      targets.data_ptr(), old.data_ptr(), None, adv.data_ptr(), 0.2,
                                                      0.2, 0.0, 1, at, at + 4, at + 16, arr, len(g),
                                                      torch.cuda.current_stream().cuda_stream))
    step(grads, out[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(other, out[1])
    emb = "transformer.wte.weight" if family == "gpt2" else "model.embed_tokens.weight"
    for k in range(3):
        flat.copy_(torch.randint(0, shape["vocab_size"], flat.shape, dtype=torch.int32))
        adv.normal_()
        step(grads, out[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1])
        for name in grads:
            if name == emb:
                assert float((grads[name] - other[name]).abs().max()) <= 1e-5 * float(grads[name].abs().max())
            else:
                assert torch.equal(grads[name], other[name]), (k, name)
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_step_on_another_stream(family):
    """The bits of the same step on the current stream, whose own work goes on."""
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 93)
    old = torch.full((len(tg),), -6.5, device="cuda")
    adv = torch.randn(len(tg), device="cuda")
    want = [t.clone() for t in m.policy_loss_and_grads(flat, cu, targets, grads, old, adv)]
    pref = [t.clone() for t in m.preference_loss_and_grads(flat, cu, targets, grads)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = m.policy_loss_and_grads(flat, cu, targets, grads, old, adv, stream=stream)
        more = m.preference_loss_and_grads(flat, cu, targets, grads, stream=stream)
        junk = [torch.full((1 << 16,), 7.0, device="cuda") for _ in range(8)]
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want + pref, (*got, *more)))
        assert all(bool((j == 7).all()) for j in junk)
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_steps_that_count_nothing(family):
    """Every gradient is overwritten with zeros; what the positions' other inputs hold
    is not used; a preference loss of equal margins is log 2."""
    shape, lens = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 102)
    none = torch.where(targets % 2 == 0, -1, shape["vocab_size"]).to(torch.int32)
    nan = torch.full((len(tg),), float("nan"), device="cuda")
    for per in (False, True):
        loss, stats, logps = m.policy_loss_and_grads(flat, cu, none, grads, nan, nan, nan, kl_coef=0.1,
                                                     per_sequence=per)
        assert not loss.any() and not stats.any() and not logps.any()
        assert all(not g.any() for g in grads.values())
    for g in grads.values():
        g.fill_(float("nan"))
    loss, seq, margins = m.preference_loss_and_grads(flat, cu, none, grads)
    assert abs(float(loss) - math.log(2)) <= 2.0 ** -23 and not seq.any() and not margins.any()
    assert all(not g.any() for g in grads.values())
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_step_of_one_token(family):
    """One sequence of one token.  Its attention has one key, so the gradients of q and k
    are zero but for the rounding of what is stored, and are left out here."""
    shape, _ = FAMILIES[family]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, [1], 105)
    targets.fill_(17)
    want, ref = ag.loss_and_grads(shape, w, seqs, ag.cross_entropy(np.array([17])))
    loss = m.loss_and_grads(flat, cu, targets, grads)
    assert abs(float(loss) - want) <= 6 * 3e-3
    assert all(bool(torch.isfinite(g).all()) for g in grads.values())
    for name, r in ref.items():
        if not any(k in name for k in ("q_proj", "k_proj", "c_attn")):
            check_weighted(name, grads[name].cpu().double().numpy(), r)
    # A = 1 and a ratio of 1: the cross-entropy's gradient, up to elements of the logits'
    # whose bf16 rounding falls the other way (2^-8)
    first = {k: g.clone() for k, g in grads.items()}
    old = -loss.clone()
    loss, stats, logps = m.policy_loss_and_grads(flat, cu, targets, grads, old, torch.ones_like(old))
    assert abs(float(loss) + 1) <= 1e-4 and abs(float(logps) - float(old)) <= 1e-4
    for name, g in grads.items():
        assert float((g - first[name]).norm()) <= 1e-2 * float(first[name].norm()) + 1e-6, name
    m.close()


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_decode_goes_on_after_a_step(family):
    """A step leaves its sequences in the cache, as a prompt would."""
    shape, lens = FAMILIES[family]
    w = model_weights(shape, seed=108)
    ids = prompts(len(lens), max(lens), shape["vocab_size"], seed=109).numpy()
    seqs = [ids[i, :n] for i, n in enumerate(lens)]
    m, fresh = (gpu_model(shape, w, max_batch=len(lens), max_seq=max(lens) + 3) for _ in range(2))
    flat, cu = pack(seqs)
    targets = torch.as_tensor(np.concatenate(_targets(seqs, shape["vocab_size"], seed=110)), dtype=torch.int32).cuda()
    grads = {k: torch.empty(tuple(v.shape), dtype=torch.float32, device="cuda") for k, v in w.items()}
    m.policy_loss_and_grads(flat, cu, targets, grads, torch.zeros(len(flat), device="cuda"),
                            torch.zeros(len(flat), device="cuda"))
    _, nxt = fresh.prefill(flat, cu)
    a, b = (torch.empty(len(lens), shape["vocab_size"], device="cuda") for _ in range(2))
    for _ in range(3):
        m.decode_step(nxt, logits=a)
        _, more = fresh.decode_step(nxt, logits=b)
        # each within 6 x 3e-3 of the exact ones
        assert float((a - b).abs().max()) <= 2 * 6 * 3e-3
        nxt = more.clone()
    m.close()
    fresh.close()


def test_refusals_of_a_step():
    shape, lens = FAMILIES["gpt2"]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 99)
    f = torch.zeros(len(tg), device="cuda")
    with pytest.raises(ValueError, match="pairs"):
        m.preference_loss_and_grads(flat[:cu[3]], cu[:4], targets, grads)
    with pytest.raises(ax.AxonError, match="kl_coef"):
        m.policy_loss_and_grads(flat, cu, targets, grads, f, f, kl_coef=0.5)
    with pytest.raises(ax.AxonError, match="beta"):
        m.preference_loss_and_grads(flat, cu, targets, grads, beta=-1.0)
    with pytest.raises(ValueError, match="old_logps"):
        m.policy_loss_and_grads(flat, cu, targets, grads, f[:3], f)
    with pytest.raises(ValueError, match="tensors on"):
        m.policy_loss_and_grads(flat, cu, targets, grads, f.cpu(), f)
    with pytest.raises(ValueError, match="gradient buffer on cpu"):
        m.policy_loss_and_grads(flat, cu, targets, {**grads, "transformer.ln_f.bias": f.cpu()}, f, f)
    with pytest.raises(ValueError, match="targets must hold"):
        m.policy_loss_and_grads(flat, cu, targets.long(), grads, f, f)
    with pytest.raises(ValueError, match="not contiguous"):
        wide = torch.empty(grads["transformer.wpe.weight"].shape[::-1], device="cuda").t()
        m.policy_loss_and_grads(flat, cu, targets, {**grads, "transformer.wpe.weight": wide}, f, f)

    class Elsewhere:  # a stream of another device
        cuda_stream, device = 0, torch.device("cuda", 1)
    with pytest.raises(ValueError, match="the stream on"):
        m.policy_loss_and_grads(flat, cu, targets, grads, f, f, stream=Elsewhere())
    with pytest.raises(ValueError, match="the stream on"):
        ops.layernorm(f.view(1, -1), f, stream=Elsewhere())
    bad = dict(grads)
    del bad["transformer.wpe.weight"]
    with pytest.raises(ax.AxonError, match="missing gradient"):
        m.loss_and_grads(flat, cu, targets, bad)
    m.close()
    paged = gpu_model(shape, w, max_batch=4, max_seq=80, page_size=16, num_pages=40)
    with pytest.raises(ax.AxonError, match="backward pass covers"):
        paged.policy_loss_and_grads(flat, cu, targets, grads, f, f)
    paged.close()
