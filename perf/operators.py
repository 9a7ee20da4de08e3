"""The row operators of a training step, as cases that can be timed: layer norm
forward and backward, the log-probabilities of given tokens and their gradient,
the preference loss over pairs of sequences and the clipped policy loss, both
with the gradient at the logits.

``run`` computes a case in its plain form (elementary torch operations in
float32, sums over sequences in float64), or, with ``own`` set, through the
public functions of ``paper_2608_19889_amd``.  Shapes are those of this
repository's models (GPT-2 XL rows of 1600 features and its odd vocabulary of
50257, the 1B shape's 128256, the 7B shape's 152064, 32000) and generic ones.
"""
import math
import random

import torch

own = False
DEV = "cuda"
EPS = 1e-5
BETA, SMOOTHING = 0.1, 0.1
CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_calls = None


def _own_calls():
    global _calls
    if _calls is None:
        import paper_2608_19889_amd as calls
        _calls = calls
    return _calls


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the rows of one GPT-2 XL decode step at batch 8: float32 residual in, bf16 operand out; latency
        dict(name="ln_fwd_decode", op="layernorm", rows=8, cols=1600, x="f32", y="bf16", pad=0),
        # a large prefill or training batch of the widest rows GPT-2 models may have here
        dict(name="ln_fwd_wide", op="layernorm", rows=16384, cols=8192, x="bf16", y="bf16", pad=0),
        # a ragged handful of rows of odd width inside a wider buffer: no 16-byte alignment anywhere
        dict(name="ln_bwd_odd", op="layernorm_backward", rows=93, cols=771, x="bf16", y="bf16", pad=6),
        # a GPT-2 XL training step of 8 x 1024 tokens: float32 residual and gradient, bf16 operand gradient
        dict(name="ln_bwd_train", op="layernorm_backward", rows=8192, cols=1600, x="f32", y="bf16", pad=0),
        # scoring three short answers with GPT-2's odd vocabulary: rows that start at any 4-byte address
        dict(name="logprobs_score", op="token_logprobs", tokens=580, seqs=3, vocab=50257, ld=50257, logits="f32"),
        # a reference model's pass over a training batch of the 1B shape (8 x 512)
        dict(name="logprobs_batch", op="token_logprobs", tokens=4096, seqs=8, vocab=128256, ld=128256, logits="f32"),
        # a caller's own loss over one short sequence
        dict(name="logprobs_bwd_short", op="token_logprobs_backward", tokens=33, seqs=1, vocab=32000, ld=32000,
             logits="bf16"),
        # the same over a batch of the 7B shape's vocabulary
        dict(name="logprobs_bwd_batch", op="token_logprobs_backward", tokens=2048, seqs=4, vocab=152064, ld=152064,
             logits="bf16"),
        # one pair of short answers
        dict(name="preference_pair", op="preference_loss", tokens=61, seqs=2, vocab=32000, ld=32000, logits="bf16"),
        # 4 pairs of about 512 tokens of the 1B shape in float32, as its logits projection leaves them
        dict(name="preference_batch", op="preference_loss", tokens=4096, seqs=8, vocab=128256, ld=128256,
             logits="f32"),
        # two short samples with GPT-2's vocabulary
        dict(name="policy_short", op="policy_loss", tokens=47, seqs=2, vocab=50257, ld=50272, logits="f32",
             per_sequence=False),
        # a group of 16 samples of one prompt, about 256 tokens each, averaged per sequence
        dict(name="policy_group", op="policy_loss", tokens=4096, seqs=16, vocab=128256, ld=128256, logits="bf16",
             per_sequence=True),
    ]


#: bytes and values of the largest listed case (preference_batch)
MOST_VALUES = 4096 * 128256


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: rows from one to 16384, widths from 64
    to 8192, vocabularies from 500 to 152064, odd values and padded rows among
    them, every type."""
    op = rng.choice(["layernorm", "layernorm_backward", "token_logprobs", "token_logprobs_backward",
                     "preference_loss", "policy_loss"])
    if op.startswith("layernorm"):
        cols = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            cols = (cols + 7) // 8 * 8
        x, y = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
        return dict(op=op, rows=_log_int(rng, 1, 16384), cols=cols, x=x, y=y, pad=rng.choice([0, 0, 8, 3]))
    vocab = _log_int(rng, 500, 152064)
    if rng.random() < 0.5:
        vocab = (vocab + 31) // 32 * 32
    ld = vocab if rng.random() < 0.7 else (vocab + 31) // 32 * 32
    tokens = min(_log_int(rng, 8, 4096), MOST_VALUES // ld)
    logits = rng.choice(["f32", "bf16"])
    seqs = rng.randint(1, max(1, min(16, tokens // 4)))
    case = dict(op=op, tokens=tokens, seqs=seqs, vocab=vocab, ld=ld, logits=logits)
    if op == "preference_loss":
        case["seqs"] = max(2, seqs // 2 * 2)
    if op == "policy_loss":
        case["per_sequence"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs

def _lens(case):
    """Sequence lengths: part of the case, so that every seed is the same work."""
    n, b = case["tokens"], case["seqs"]
    r = random.Random("%d %d %d" % (n, b, case["vocab"]))
    share = [r.uniform(0.6, 1.4) for _ in range(b)]
    lens = [max(1, int(n * s / sum(share))) for s in share]
    lens[-1] += n - sum(lens)
    return lens if lens[-1] >= 1 else [n - (b - 1)] + [1] * (b - 1)


def _counted(case):
    """Whether each position counts: none at a sequence's end (it has no next
    token) and, for the two losses, none in the first third (the prompt)."""
    out = []
    for n in _lens(case):
        first = n // 3 if case["op"] in ("preference_loss", "policy_loss") else 0
        out += [first <= i < n - 1 for i in range(n)]
    return out


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _padded(t, pad, dtype):
    """``t`` as a view of rows that lie ``pad`` values further apart."""
    if not pad:
        return t.to(dtype)
    wide = torch.zeros((t.shape[0], t.shape[1] + pad), device=DEV, dtype=dtype)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & ((1 << 62) - 1))
    st = dict(case=case)
    if case["op"].startswith("layernorm"):
        R, C = case["rows"], case["cols"]
        # residual rows: a common offset, a few large features, rows of different size
        x = _randn(g, R, C) * (0.5 + 2 * torch.rand((R, 1), generator=g, device=DEV)) + 0.3 * _randn(g, 1, C)
        st["x"] = _padded(x, case["pad"], TYPES[case["x"]])
        par = TYPES[case["y"]]
        st["gain"] = (1 + 0.1 * _randn(g, C)).to(par)
        st["bias"] = (0.1 * _randn(g, C)).to(par)
        if case["op"] == "layernorm_backward":
            st["dy"] = _padded(_randn(g, R, C), case["pad"], TYPES[case["y"]])
        return st
    T, V, ld = case["tokens"], case["vocab"], case["ld"]
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int64)
    z = _randn(g, T, ld).mul_(2.0)
    # a trained model gives the tokens it is shown more than the others
    z[torch.arange(T, device=DEV), targets] += 10 * torch.rand((T,), generator=g, device=DEV)
    z = z.to(TYPES[case["logits"]])
    st["logits"] = z[:, :V]
    counted = torch.tensor(_counted(case), device=DEV)
    st["targets"] = torch.where(counted, targets, torch.full_like(targets, -1)).to(torch.int32)
    cu = [0]
    for n in _lens(case):
        cu.append(cu[-1] + n)
    st["cu"] = cu
    st["cu_device"] = torch.tensor(cu, dtype=torch.int32, device=DEV)
    st["seq"] = torch.repeat_interleave(torch.arange(len(cu) - 1, device=DEV),
                                        torch.tensor(_lens(case), device=DEV))
    if case["op"] == "token_logprobs_backward":
        st["dlogps"] = _randn(g, T) / T
    if case["op"] in ("preference_loss", "policy_loss"):
        logps = _plain_logps(st["logits"], st["targets"])
        if case["op"] == "preference_loss":
            # a reference from which the policy has begun to move
            sums = torch.zeros(len(cu) - 1, dtype=torch.float64, device=DEV).index_add_(0, st["seq"], logps.double())
            st["ref"] = (sums + 8 * _randn(g, len(cu) - 1).double()).float()
        else:
            moved = 0.2 * _randn(g, T)
            # no ratio within a thousandth of where it is clipped: there a last digit decides about a whole row
            for edge in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
                moved = torch.where((moved - edge).abs() < 1e-3, moved + 3e-3, moved)
            st["old"] = logps - moved
            st["ref"] = logps + 0.4 * _randn(g, T)
            st["adv"] = 0.7 * _randn(g, T) + 1
            # what stands at positions that do not count is never used
            st["old"][~counted] = float("nan")
            st["adv"][~counted] = float("inf")
    return st


# ------------------------------------------------------------------ plain forms

def _plain_ln(x, gain, bias, out):
    xf = x.float()
    d = xf - xf.sum(-1, keepdim=True) / x.shape[1]
    var = (d * d).sum(-1, keepdim=True) / x.shape[1]
    return (d * torch.rsqrt(var + EPS) * gain.float() + bias.float()).to(out)


def _plain_ln_backward(dy, x, gain):
    C = x.shape[1]
    xf, dyf = x.float(), dy.float()
    d = xf - xf.sum(-1, keepdim=True) / C
    rstd = torch.rsqrt((d * d).sum(-1, keepdim=True) / C + EPS)
    xhat = d * rstd
    gdy = dyf * gain.float()
    dx = rstd * (gdy - gdy.sum(-1, keepdim=True) / C - xhat * ((gdy * xhat).sum(-1, keepdim=True) / C))
    return dx.to(x.dtype), (dyf * xhat).sum(0), dyf.sum(0)


def _plain_rows(logits, targets):
    """(log-probability of each target in 64 bits, 0 where it does not count;
    counted; largest logit; sum of exponentials)"""
    z = logits.float()
    top = z.max(-1, keepdim=True).values
    total = torch.exp(z - top).sum(-1, keepdim=True)
    ok = (targets >= 0) & (targets < logits.shape[1])
    at = torch.where(ok, targets, torch.zeros_like(targets)).long()
    # a ratio of two probabilities shows every digit of their logarithms: 64 bits from here
    lp = z.gather(1, at[:, None]).double() - top.double() - torch.log(total.double())
    return torch.where(ok, lp[:, 0], torch.zeros_like(lp[:, 0])), ok, top, total


def _plain_logps(logits, targets):
    return _plain_rows(logits, targets)[0].float()


def _plain_grad(logits, targets, ok, top, total, dlogps):
    """sum_t dlogps[t] * d logps[t] / d logits"""
    w = torch.where(ok, dlogps, torch.zeros_like(dlogps))[:, None]
    d = torch.exp(logits.float() - top) / total * -w
    at = torch.where(ok, targets, torch.zeros_like(targets)).long()
    d.scatter_add_(1, at[:, None], w)
    return d.to(logits.dtype)


def _plain_preference(st):
    z, tg, seq = st["logits"], st["targets"], st["seq"]
    lp, ok, top, total = _plain_rows(z, tg)
    n = len(st["cu"]) - 1
    sums = torch.zeros(n, dtype=torch.float64, device=z.device).index_add_(0, seq, lp)
    r = sums - st["ref"].double()
    u = BETA * (r[0::2] - r[1::2])
    softplus = lambda v: torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
    loss = ((1 - SMOOTHING) * softplus(-u) + SMOOTHING * softplus(u)).sum() / (n // 2)
    sig = 1 / (1 + torch.exp(-u))
    du = (SMOOTHING * sig - (1 - SMOOTHING) * (1 - sig)) / (n // 2)
    ds = torch.stack([BETA * du, -BETA * du], 1).reshape(-1)
    return dict(loss=loss.float().reshape(1), seq_logps=sums.float(), margins=u.float(),
                dlogits=_plain_grad(z, tg, ok, top, total, ds[seq].float()))


def _plain_policy(st):
    z, tg, seq = st["logits"], st["targets"], st["seq"]
    lp, ok, top, total = _plain_rows(z, tg)
    zero = torch.zeros_like(lp)
    old, ref, adv = (torch.where(ok, st[k].double(), zero) for k in ("old", "ref", "adv"))
    if st["case"]["per_sequence"]:
        n = torch.zeros(len(st["cu"]) - 1, dtype=torch.float64, device=z.device).index_add_(0, seq, ok.double())
        w = 1 / torch.clamp(n, min=1)[seq] / torch.clamp((n > 0).sum(), min=1)
    else:
        w = torch.ones_like(lp) / torch.clamp(ok.sum(), min=1)
    w = torch.where(ok, w, zero)
    ratio = torch.exp(lp - old)
    held = torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH)
    free = ratio * adv <= held * adv
    surrogate = -torch.minimum(ratio * adv, held * adv)
    gap = ref - lp
    kl = torch.exp(gap) - gap - 1
    dlp = w * (torch.where(free, -ratio * adv, zero) + KL_COEF * (1 - torch.exp(gap)))
    mean = lambda v: (w * v).sum()  # noqa: E731
    stats = torch.stack([mean(surrogate), mean(kl), mean((~free).double())]).float()
    return dict(loss=mean(surrogate + KL_COEF * kl).float().reshape(1), stats=stats, logps=lp.float(),
                dlogits=_plain_grad(z, tg, ok, top, total, dlp.float()))


def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(op, st)
    if op == "layernorm":
        return _plain_ln(st["x"], st["gain"], st["bias"], TYPES[st["case"]["y"]])
    if op == "layernorm_backward":
        return dict(zip(("dx", "dgain", "dbias"), _plain_ln_backward(st["dy"], st["x"], st["gain"])))
    if op == "token_logprobs":
        return _plain_logps(st["logits"], st["targets"])
    if op == "token_logprobs_backward":
        _, ok, top, total = _plain_rows(st["logits"], st["targets"])
        return _plain_grad(st["logits"], st["targets"], ok, top, total, st["dlogps"])
    return _plain_preference(st) if op == "preference_loss" else _plain_policy(st)


def _run_own(op, st):
    c = _own_calls()
    if op == "layernorm":
        return c.layernorm(st["x"], st["gain"], st["bias"], EPS, dtype=TYPES[st["case"]["y"]])
    if op == "layernorm_backward":
        return dict(zip(("dx", "dgain", "dbias"), c.layernorm_backward(st["dy"], st["x"], st["gain"], EPS)))
    if op == "token_logprobs":
        return c.token_logprobs(st["logits"], st["targets"])
    if op == "token_logprobs_backward":
        return c.token_logprobs_backward(st["logits"], st["targets"], st["dlogps"])
    if op == "preference_loss":
        got = c.preference_loss(st["logits"], st["targets"], st["cu"], ref_logps=st["ref"], beta=BETA,
                                label_smoothing=SMOOTHING, cu_device=st["cu_device"])
        return dict(zip(("loss", "seq_logps", "margins", "dlogits"), got))
    got = c.policy_loss(st["logits"], st["targets"], st["cu"], st["old"], st["adv"], ref_logps=st["ref"],
                        clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF,
                        per_sequence=st["case"]["per_sequence"], cu_device=st["cu_device"])
    return dict(zip(("loss", "stats", "logps", "dlogits"), got))


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"].startswith("layernorm"):
        n, x, y = case["rows"] * case["cols"], size[case["x"]], size[case["y"]]
        if case["op"] == "layernorm":
            return {"bytes": n * (x + y) + 2 * case["cols"] * y, "flops": 8 * n}
        return {"bytes": n * (2 * x + y) + case["cols"] * (y + 8), "flops": 16 * n}
    # the logits of positions that count are read; their gradient is written at every position
    V, e = case["vocab"], size[case["logits"]]
    read = sum(_counted(case)) * V * e
    wrote = 0 if case["op"] == "token_logprobs" else case["tokens"] * V * e
    return {"bytes": read + wrote + 12 * case["tokens"], "flops": 3 * sum(_counted(case)) * V * (2 if wrote else 1)}


# ------------------------------------------------------------------ 64 bits

def _exact_rows(z, tg, dlogps=None):
    """Log-probabilities (0 where a target does not count) and, with a function
    of them for each position's weight, the gradient; 256 rows at a time."""
    T, V = z.shape
    ok = (tg >= 0) & (tg < V)
    lp = torch.zeros(T, dtype=torch.float64, device=z.device)
    for i in range(0, T, 256):
        rows = z[i:i + 256].double()
        part = torch.log_softmax(rows, -1)
        lp[i:i + 256] = part[torch.arange(len(rows), device=z.device), tg[i:i + 256].long().clamp(0, V - 1)]
    lp[~ok] = 0
    if dlogps is None:
        return lp, None
    w = dlogps(lp, ok)
    grad = torch.zeros((T, V), dtype=torch.float64, device=z.device)
    for i in range(0, T, 256):
        c, r = ok[i:i + 256], torch.arange(len(z[i:i + 256]), device=z.device)
        g = torch.softmax(z[i:i + 256].double(), -1).neg_()
        g[r, tg[i:i + 256].long().clamp(0, V - 1)] += 1
        grad[i:i + 256] = torch.where(c[:, None], w[i:i + 256, None] * g, 0.0)
    return lp, grad


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op.startswith("layernorm"):
        dx, y, C = [], [], case["cols"]
        g, b = st["gain"].double(), st["bias"].double()
        dgain, dbias = torch.zeros_like(g), torch.zeros_like(g)
        for i in range(0, case["rows"], 1024):
            x = st["x"][i:i + 1024].double()
            sd = torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS)
            xhat = (x - x.mean(-1, keepdim=True)) / sd
            if op == "layernorm":
                y.append(xhat * g + b)
                continue
            dy = st["dy"][i:i + 1024].double()
            dgain += (dy * xhat).sum(0)
            dbias += dy.sum(0)
            h = dy * g
            dx.append((h - h.mean(-1, keepdim=True) - xhat * (h * xhat).mean(-1, keepdim=True)) / sd)
        return torch.cat(y) if op == "layernorm" else dict(dx=torch.cat(dx), dgain=dgain, dbias=dbias)
    z, tg, cu = st["logits"], st["targets"], st["cu"]
    if op == "token_logprobs":
        return _exact_rows(z, tg)[0]
    if op == "token_logprobs_backward":
        return _exact_rows(z, tg, lambda lp, ok: st["dlogps"].double())[1]
    got = {}
    if op == "preference_loss":
        def weights(lp, ok):
            s = torch.stack([lp[a:b].sum() for a, b in zip(cu, cu[1:])])
            gap = (s - st["ref"].double()).reshape(-1, 2)
            u = BETA * (gap[:, 0] - gap[:, 1])
            yes = torch.nn.functional.logsigmoid(u)
            no = torch.nn.functional.logsigmoid(-u)
            got.update(seq_logps=s, margins=u, loss=-((1 - SMOOTHING) * yes + SMOOTHING * no).mean().reshape(1))
            du = -((1 - SMOOTHING) * no.exp() - SMOOTHING * yes.exp()) / len(u) * BETA
            return torch.cat([du[i // 2].expand(b - a) * (1 - 2 * (i % 2)) for i, (a, b) in enumerate(zip(cu, cu[1:]))])
    else:
        def weights(lp, ok):
            w = torch.zeros_like(lp)
            if case["per_sequence"]:
                full = [(a, b) for a, b in zip(cu, cu[1:]) if bool(ok[a:b].any())]
                for a, b in full:
                    w[a:b] = 1 / ok[a:b].sum().double() / len(full)
            else:
                w[:] = 1 / ok.sum().clamp(min=1).double()
            w[~ok] = 0
            old, ref, adv = (torch.where(ok, st[k].double(), 0.0) for k in ("old", "ref", "adv"))
            q = torch.exp(lp - old)
            stopped = ((adv > 0) & (q > 1 + CLIP_HIGH)) | ((adv < 0) & (q < 1 - CLIP_LOW))
            term = -adv * torch.where(stopped, q.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH), q)
            kl = torch.expm1(ref - lp) - (ref - lp)
            got.update(logps=lp, loss=(w * (term + KL_COEF * kl)).sum().reshape(1),
                       stats=torch.stack([(w * term).sum(), (w * kl).sum(), (w * stopped).sum()]))
            return w * (torch.where(stopped, 0.0, -adv * q) - KL_COEF * torch.expm1(ref - lp))
    _, got["dlogits"] = _exact_rows(z, tg, weights)
    return got
