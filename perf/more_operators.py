"""The operators that sample a group of answers to a prompt, as cases that can be
timed: rotating queries and keys and appending keys and values to a paged cache,
attention over that cache for sequences that share a long prefix, and drawing the
next tokens from given random numbers.

``run`` computes a case in its plain form (elementary torch operations in float32;
angles, exponentials and sums of a distribution in float64), or, with ``own`` set,
through the public functions of ``paper_2608_19889_amd``.  Head layouts and
vocabularies are those of this repository's models (135M: 9 heads over 3 of 64,
49152; 1B: 32 over 8 of 64, 128256; 7B: 28 over 4 of 128, 152064; 32B: 40 over 8 of
128; GPT-2 XL: 25 of 64, 50257; 32000) and generic ones.
"""
import math
import random

import torch

own = False
DEV = "cuda"
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
        # one decode step of the 1B workload (8 sequences), its theta: latency
        dict(name="append_decode", op="append", heads=32, kv=8, hd=64, type="bf16", page=16, seqs=8, new=1, past=600,
             prefix=0, theta=500000.0, rot=64, interleaved=False, fused=False),
        # 12 prompts of the 7B shape enter the cache in one ragged call, out of one fused projection
        dict(name="append_prompts", op="append", heads=28, kv=4, hd=128, type="bf16", page=16, seqs=12, new=1400,
             past=0, prefix=0, theta=1000000.0, rot=128, interleaved=False, fused=True),
        # chunks behind a long shared document, half of each head rotated pair by pair: far angles, odd counts
        dict(name="append_far", op="append", heads=9, kv=3, hd=64, type="f32", page=48, seqs=7, new=101, past=333,
             prefix=700001, theta=10000.0, rot=32, interleaved=True, fused=True),
        # four answers to a short question in the 135M shape's float32: latency
        dict(name="attend_few", op="attend", heads=9, kv=3, hd=64, type="f32", page=16, groups=1, seqs=4, new=1,
             prefix=300, past=40),
        # 64 answers to one prompt of the 7B shape, as a policy step samples them
        dict(name="attend_group", op="attend", heads=28, kv=4, hd=128, type="bf16", page=16, groups=1, seqs=64, new=1,
             prefix=4096, past=600),
        # 16 prompts of different length with 16 answers each, 1B shape
        dict(name="attend_groups", op="attend", heads=32, kv=8, hd=64, type="bf16", page=32, groups=16, seqs=16, new=1,
             prefix=1100, past=300),
        # 48 answers to a question about a long document, 32B shape
        dict(name="attend_long", op="attend", heads=40, kv=8, hd=128, type="bf16", page=64, groups=1, seqs=48, new=1,
             prefix=50011, past=900),
        # ragged questions of some hundred tokens behind one system prompt, 7B shape: many new tokens a sequence
        dict(name="attend_questions", op="attend", heads=28, kv=4, hd=128, type="bf16", page=16, groups=1, seqs=20,
             new=150, prefix=2500, past=0),
        # a small batch of 32000 tokens' logits, the usual two filters: latency
        dict(name="sample_few", op="sample", rows=8, vocab=32000, ld=32000, type="f32", filters="k+p"),
        # a group of 64 answers with the 7B shape's vocabulary and a nucleus
        dict(name="sample_nucleus", op="sample", rows=64, vocab=152064, ld=152064, type="f32", filters="p"),
        # GPT-2's odd vocabulary in bf16, the whole distribution: what a policy step samples from
        dict(name="sample_whole", op="sample", rows=93, vocab=50257, ld=50272, type="bf16", filters="none"),
        # a large serving batch in which every request has its own settings, some of them a grammar's mask
        dict(name="sample_mixed", op="sample", rows=384, vocab=128256, ld=128256, type="f32", filters="mixed"),
    ]


HEADS = [(9, 3, 64), (32, 8, 64), (28, 4, 128), (40, 8, 128), (25, 25, 64), (16, 16, 128), (32, 8, 128), (12, 1, 64)]
#: what the largest listed case of each kind reads and writes (bytes) and computes (operations)
MOST = {"append": 307e6, "attend": 375e6, "sample": 197e6}
MOST_FLOPS = 100e9


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["append", "attend", "sample"])
    if op == "sample":
        vocab = _log_int(rng, 500, 152064)
        if rng.random() < 0.5:
            vocab = (vocab + 31) // 32 * 32
        ld = vocab if rng.random() < 0.7 else (vocab + 31) // 32 * 32
        return dict(op=op, rows=_log_int(rng, 1, 512), vocab=vocab, ld=ld, type=rng.choice(["f32", "bf16"]),
                    filters=rng.choice(["none", "k", "p", "k+p", "min", "mixed"]))
    heads, kv, hd = rng.choice(HEADS)
    case = dict(op=op, heads=heads, kv=kv, hd=hd, type=rng.choice(["bf16", "bf16", "f32"]),
                page=rng.choice([16, 32, 48, 64, 128]))
    if op == "append":
        case.update(seqs=_log_int(rng, 1, 64), new=rng.choice([1, _log_int(rng, 2, 2000)]),
                    past=rng.choice([0, _log_int(rng, 1, 2000)]), prefix=rng.choice([0, _log_int(rng, 100, 1000000)]),
                    theta=rng.choice([10000.0, 500000.0, 1000000.0]), rot=rng.choice([hd, hd, hd // 2, hd // 4]),
                    interleaved=rng.random() < 0.4, fused=rng.random() < 0.5)
    else:
        case.update(groups=_log_int(rng, 1, 16), seqs=_log_int(rng, 1, 64), new=rng.choice([1, 1, _log_int(rng, 2, 200)]),
                    prefix=_log_int(rng, 1, 50000), past=rng.choice([0, _log_int(rng, 1, 2000)]))
    return case


def draw(rng):
    """One more case of the same ranges: one sequence to hundreds, one new token to
    thousands, prefixes and pasts of one token to tens of thousands, every head layout,
    type, page size and filter, vocabularies from 500 to 152064, odd values among them."""
    while True:
        case = _draw(rng)
        w = work(case)
        cached = sum(_prefixes(case)) + sum(_pasts(case)) + sum(_news(case)) if case["op"] != "sample" else 0
        if w["bytes"] <= MOST[case["op"]] and w["flops"] <= MOST_FLOPS and cached <= 120000:
            return case


# ------------------------------------------------------------------ inputs

def _spread(case, what, n, mean, least):
    """n lengths about ``mean``: part of the case, so that every seed is the same work."""
    r = random.Random("%s %d %d %d" % (what, n, mean, case["heads"]))
    return [max(least, int(round(mean * r.uniform(0.3, 1.7)))) if mean > 1 else mean for _ in range(n)]


def _groups(case):
    return case.get("groups", 1)


def _prefixes(case):
    if _groups(case) == 1:
        return [case["prefix"]]
    return _spread(case, "prefix", _groups(case), case["prefix"], 1)


def _pasts(case):
    return _spread(case, "past", _groups(case) * case["seqs"], case["past"], 0)


def _news(case):
    return _spread(case, "new", _groups(case) * case["seqs"], case["new"], 1)


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _tables(g, page, *lens):
    """Page tables for lists of sequences, their pages in random order in one pool:
    (pages of the pool, a device int32 [sequences, most pages] for each list)."""
    counts = [[-(-n // page) for n in group] for group in lens]
    pool = max(1, sum(map(sum, counts)))
    ids = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    tables, at = [], 0
    for group in counts:
        t = torch.full((len(group), max([1, *group])), -1, dtype=torch.int32, device=DEV)
        for i, n in enumerate(group):
            t[i, :n] = ids[at:at + n]
            at += n
        tables.append(t)
    return pool, tables


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _heads(case, g, tokens):
    """q, k, v [tokens, heads, hd], of one fused projection or each for itself."""
    H, KV, hd, t = case["heads"], case["kv"], case["hd"], TYPES[case["type"]]
    if case.get("fused"):
        rows = _randn(g, tokens, H + 2 * KV, hd).to(t)
        return rows[:, :H], rows[:, H:H + KV], rows[:, H + KV:]
    return tuple(_randn(g, tokens, n, hd).to(t) for n in (H, KV, KV))


def _filters(case, g, rows):
    kind = case["filters"]
    if kind == "mixed":
        pick = torch.randint(0, 5, (rows,), generator=g, device=DEV)
        u = torch.rand((4, rows), generator=g, device=DEV)
        on = lambda *which: sum((pick == i) for i in which) > 0  # noqa: E731
        return dict(temperature=torch.where(pick == 4, 0.0, 0.3 + 1.0 * u[0]).float(),
                    top_k=torch.where(on(0, 1), (1 + 80 * u[1]).int(), 0).to(torch.int32),
                    top_p=torch.where(on(1, 2), 0.5 + 0.49 * u[2], 1.0).float(),
                    min_p=torch.where(on(2, 3), 0.01 + 0.1 * u[3], 0.0).float())
    return {"none": dict(temperature=1.0), "k": dict(temperature=0.7, top_k=50), "p": dict(temperature=0.8, top_p=0.95),
            "k+p": dict(temperature=0.8, top_k=40, top_p=0.9), "min": dict(temperature=1.3, min_p=0.05)}[kind]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & ((1 << 62) - 1))
    st = dict(case=case)
    if case["op"] == "sample":
        R, V, ld = case["rows"], case["vocab"], case["ld"]
        # a trained model's logits: a broad bulk and some hundred tokens that fit, falling with their rank; most
        # rows are sure of themselves, some leave much to the bulk
        z = _randn(g, R, ld).mul_(1.5)
        n = min(V, 400)
        step = next(s for s in range(int(0.618 * V), V) if math.gcd(s, V) == 1)  # n different places of each row
        first = torch.randint(0, V, (R, 1), generator=g, device=DEV)
        at = (first + step * torch.arange(n, device=DEV)) % V
        top = 13 + 8 * torch.rand((R, 1), generator=g, device=DEV) - math.log(152064 / V)
        fall = 1 + torch.rand((R, 1), generator=g, device=DEV)
        z.scatter_(1, at, top - fall * torch.log1p(torch.arange(n, device=DEV)) + 0.3 * _randn(g, R, n))
        if case["filters"] == "mixed":
            # a grammar leaves every 16th row few tokens
            few = torch.rand((len(range(5, R, 16)), ld), generator=g, device=DEV) > 20 / V
            few[:, V // 2] = False
            z[5::16] = torch.where(few, float("-inf"), z[5::16])
        st["logits"] = z.to(TYPES[case["type"]])[:, :V]
        st["uniform"] = torch.rand((R,), generator=g, device=DEV)
        st["filters"] = _filters(case, g, R)
        return st
    page, past, new = case["page"], _pasts(case), _news(case)
    dtype, H, KV, hd = TYPES[case["type"]], case["heads"], case["kv"], case["hd"]
    st["cu"] = None if all(n == 1 for n in new) else _cu(new)
    st["cu_device"] = None if st["cu"] is None else _ints(st["cu"])
    st["lens"] = _ints(past)
    T = sum(new)
    held = [p + n for p, n in zip(past, new)]
    if case["op"] == "append":
        pool, (st["table"],) = _tables(g, page, held)
        st["q"], st["k"], st["v"] = _heads(case, g, T)
        st["offsets"] = _ints([case["prefix"]] * len(past)) if case["prefix"] else None
        rot = case["rot"]
        st["inv_freq"] = case["theta"] ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
        # a context stretched over that of the training scales what it rotates
        st["scale"] = 1.0 if case["prefix"] < 100000 else 1.25
    else:
        prefix = _prefixes(case)
        pool, (st["table"], st["prefix_table"]) = _tables(g, page, held, prefix)
        st["q"] = (1.5 * _randn(g, T, H, hd)).to(dtype)
        st["prefix_lens"] = _ints(prefix)
        st["cu_groups"] = [i * case["seqs"] for i in range(len(prefix) + 1)]
        st["groups_device"] = _ints(st["cu_groups"])
    st["k_cache"], st["v_cache"] = (_randn(g, pool, KV, page, hd).to(dtype) for _ in range(2))
    if case["op"] == "attend":
        # what stands behind a sequence's last key is never used
        for table, lens in ((st["table"], held), (st["prefix_table"], prefix)):
            ends = [(i, n) for i, n in enumerate(lens) if n % page]
            if ends:
                rows, n = (torch.tensor(v, device=DEV) for v in zip(*ends))
                ids = table[rows, n // page].long()
                behind = (torch.arange(page, device=DEV) >= (n % page)[:, None])[:, None, :, None]
                for cache, junk in ((st["k_cache"], float("nan")), (st["v_cache"], float("inf"))):
                    cache[ids] = torch.where(behind, junk, cache[ids].float()).to(dtype)
    return st


# ------------------------------------------------------------------ plain forms

def _sequences(st):
    """(each token's sequence, its number there) and each sequence's first token."""
    B = st["table"].shape[0]
    if st["cu"] is None:
        first = torch.arange(B + 1, device=DEV)
    else:
        first = st["cu_device"].long()
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), first[1:] - first[:-1], output_size=st["q"].shape[0])
    return seq, torch.arange(st["q"].shape[0], device=DEV) - first[seq]


def _plain_rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    c, s = cos[:, None], sin[:, None]
    pair = (a * c - b * s, b * c + a * s)
    done = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat([done, x[..., rot:]], -1)


def _plain_append(st):
    case, page = st["case"], st["case"]["page"]
    seq, nth = _sequences(st)
    slot = st["lens"].long()[seq] + nth
    at = slot if st["offsets"] is None else slot + st["offsets"].long()[seq]
    angle = at.double()[:, None] * st["inv_freq"]
    cos, sin = (torch.cos(angle) * st["scale"]).float(), (torch.sin(angle) * st["scale"]).float()
    turn = lambda x: _plain_rotate(x, cos, sin, case["rot"], case["interleaved"]).to(x.dtype)  # noqa: E731
    ids = st["table"].long()[seq, slot // page]
    st["k_cache"][ids, :, slot % page] = turn(st["k"])
    st["v_cache"][ids, :, slot % page] = st["v"]
    return dict(q=turn(st["q"]), k_cache=st["k_cache"], v_cache=st["v_cache"])


def _gather(cache, pages, n):
    """the first n keys (or values) behind a row of pages, float32 [kv, n, hd]"""
    got = cache[pages.long()].float()
    return got.permute(1, 0, 2, 3).reshape(got.shape[1], -1, got.shape[3])[:, :n]


def _plain_part(q, k, v, seen=None):
    """(maximum, sum, product) of a softmax over some keys: q [kv, rows, hd]"""
    s = torch.matmul(q, k.transpose(1, 2).contiguous())
    if seen is not None:
        s = torch.where(seen, s, float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    return top, p.sum(-1, keepdim=True), torch.matmul(p, v)


def _plain_attend(st):
    case = st["case"]
    H, KV, hd, page = case["heads"], case["kv"], case["hd"], case["page"]
    G = H // KV
    T = st["q"].shape[0]
    cu = st["cu"] if st["cu"] is not None else list(range(T + 1))
    past, prefix = _pasts(case), _prefixes(case)
    # rows of a key/value head: its tokens' query heads
    q = (st["q"].float() / math.sqrt(hd)).view(T, KV, G, hd).permute(1, 0, 2, 3).reshape(KV, T * G, hd)
    out = torch.empty_like(q)
    for g, n in enumerate(prefix):
        pages = st["prefix_table"][g, :-(-n // page)]
        k, v = _gather(st["k_cache"], pages, n), _gather(st["v_cache"], pages, n)
        lo, hi = st["cu_groups"][g], st["cu_groups"][g + 1]
        shared = _plain_part(q[:, cu[lo] * G:cu[hi] * G], k, v)
        for b in range(lo, hi):
            new, rows = cu[b + 1] - cu[b], slice(cu[b] * G, cu[b + 1] * G)
            held = past[b] + new
            pages = st["table"][b, :-(-held // page)]
            seen = None
            if new > 1:
                at = past[b] + torch.arange(new, device=DEV).repeat_interleave(G)
                seen = torch.arange(held, device=DEV)[None, :] <= at[:, None]
            m1, l1, o1 = _plain_part(q[:, rows], _gather(st["k_cache"], pages, held),
                                     _gather(st["v_cache"], pages, held), seen)
            here = slice((cu[b] - cu[lo]) * G, (cu[b + 1] - cu[lo]) * G)
            m0, l0, o0 = (x[:, here] for x in shared)
            top = torch.maximum(m0, m1)
            a0, a1 = torch.exp(m0 - top), torch.exp(m1 - top)
            out[:, rows] = (o0 * a0 + o1 * a1) / (l0 * a0 + l1 * a1)
    return out.view(KV, T, G, hd).permute(1, 0, 2, 3).reshape(T, H, hd).to(st["q"].dtype)


def _per_row(value, rows, dtype):
    if isinstance(value, torch.Tensor):
        return value.to(dtype)[:, None]
    # a number is handed over in 32 bits
    return torch.full((rows, 1), value, dtype=torch.float32, device=DEV).to(dtype)


def _plain_sample(st):
    """Rows in descending order of their logits (the lowest index first among equals):
    each filter keeps a beginning of it; the token is where the kept weights, summed in
    the order of the vocabulary, pass ``uniform`` of their sum."""
    tokens, logps = [], []
    f = st["filters"]
    R, V = st["logits"].shape
    temperature, top_p, min_p = (_per_row(f.get(n, d), R, torch.float64)
                                 for n, d in (("temperature", 1.0), ("top_p", 1.0), ("min_p", 0.0)))
    top_k = _per_row(f.get("top_k", 0), R, torch.int64)
    for i in range(0, R, 64):
        part = slice(i, i + 64)
        z = st["logits"][part].float()
        order = torch.sort(z, dim=1, descending=True, stable=True)
        t = temperature[part]
        greedy = t <= 0
        w = torch.exp((order.values.double() - order.values[:, :1].double()) / torch.where(greedy, 1.0, t))
        rank = torch.arange(V, device=DEV)[None, :]
        k = torch.where(top_k[part] > 0, top_k[part], V)
        k = torch.where(greedy, 1, k)
        w = torch.where(rank < k, w, 0.0)
        before = torch.cumsum(w, 1) - w
        keep = (before < top_p[part] * w.sum(1, keepdim=True)) | (top_p[part] >= 1) | (rank == 0)
        keep &= (w >= min_p[part]) & (w > 0)
        w = torch.where(keep, w, 0.0)
        back = torch.zeros_like(w).scatter_(1, order.indices, w)
        total = torch.cumsum(back, 1)
        mass = total[:, -1:]
        passed = (total > st["uniform"][part, None].double() * mass) & (back > 0)
        token = passed.to(torch.int32).argmax(1, keepdim=True)
        tokens.append(token[:, 0].to(torch.int32))
        logps.append(torch.log(back.gather(1, token) / mass)[:, 0].float())
    return dict(tokens=torch.cat(tokens), logprobs=torch.cat(logps))


def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(op, st)
    return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[op](st)


def _run_own(op, st):
    c = _own_calls()
    if op == "append":
        q = c.rope_append(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lens"],
                          st["inv_freq"], cu_seqlens=st["cu"], cu_device=st["cu_device"], offsets=st["offsets"],
                          interleaved=st["case"]["interleaved"], scale=st["scale"])
        return dict(q=q, k_cache=st["k_cache"], v_cache=st["v_cache"])
    if op == "attend":
        return c.prefix_attention(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"],
                                  prefix_table=st["prefix_table"], prefix_lens=st["prefix_lens"],
                                  cu_groups=st["cu_groups"], groups_device=st["groups_device"],
                                  cu_seqlens=st["cu"], cu_device=st["cu_device"])
    tokens, logprobs = c.sample_tokens(st["logits"], st["uniform"], **st["filters"])
    return dict(tokens=tokens, logprobs=logprobs)


def work(case):
    size = {"f32": 4, "bf16": 2}[case["type"]]
    if case["op"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * size + 12), "flops": 2 * case["rows"] * case["vocab"]}
    H, KV, hd = case["heads"], case["kv"], case["hd"]
    new, past = _news(case), _pasts(case)
    T = sum(new)
    if case["op"] == "append":
        return {"bytes": T * 2 * (H + 2 * KV) * hd * size, "flops": T * 3 * (H + KV) * case["rot"]}
    seqs, pairs, keys = case["seqs"], 0, 0
    for g, n in enumerate(_prefixes(case)):
        keys += n
        for b in range(g * seqs, (g + 1) * seqs):
            keys += past[b] + new[b]
            pairs += new[b] * (n + past[b]) + new[b] * (new[b] + 1) // 2
    return {"bytes": (keys * 2 * KV + T * 2 * H) * hd * size, "flops": 4 * pairs * H * hd}


# ------------------------------------------------------------------ 64 bits

def _exact_append(st):
    case, page, rot = st["case"], st["case"]["page"], st["case"]["rot"]
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    qs = []
    cu = st["cu"] if st["cu"] is not None else list(range(len(st["lens"]) + 1))
    for b, past in enumerate(st["lens"].tolist()):
        rows = slice(cu[b], cu[b + 1])
        slots = torch.arange(past, past + cu[b + 1] - cu[b], device=DEV)
        base = 0 if st["offsets"] is None else int(st["offsets"][b])
        turn = st["scale"] * torch.exp(1j * (slots + base).double()[:, None, None] * st["inv_freq"])

        def rotated(x):
            x = x.double().clone()
            if case["interleaved"]:
                x[..., :rot] = torch.view_as_real(torch.view_as_complex(
                    x[..., :rot].reshape(*x.shape[:2], rot // 2, 2).contiguous()) * turn).flatten(-2)
            else:
                both = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
                x[..., :rot // 2], x[..., rot // 2:rot] = both.real, both.imag
            return x
        qs.append(rotated(st["q"][rows]))
        pages = st["table"][b].long()[slots // page]
        kc[pages, :, slots % page] = rotated(st["k"][rows])
        vc[pages, :, slots % page] = st["v"][rows].double()
    return dict(q=torch.cat(qs), k_cache=kc, v_cache=vc)


def _exact_attend(st):
    """Every sequence over its whole context at once, one key/value head at a time."""
    case = st["case"]
    H, KV, hd, page = case["heads"], case["kv"], case["hd"], case["page"]
    T, G = st["q"].shape[0], H // KV
    out = torch.empty((T, H, hd), dtype=torch.float64, device=DEV)
    cu = st["cu"] if st["cu"] is not None else list(range(T + 1))
    past, prefix = _pasts(case), _prefixes(case)
    for h in range(KV):
        for g, n in enumerate(prefix):
            front = [c[st["prefix_table"][g, :-(-n // page)].long(), h].reshape(-1, hd)[:n].double()
                     for c in (st["k_cache"], st["v_cache"])]
            for b in range(st["cu_groups"][g], st["cu_groups"][g + 1]):
                new = cu[b + 1] - cu[b]
                held = past[b] + new
                tail = [c[st["table"][b, :-(-held // page)].long(), h].reshape(-1, hd)[:held].double()
                        for c in (st["k_cache"], st["v_cache"])]
                k, v = (torch.cat(pair) for pair in zip(front, tail))
                rows = st["q"][cu[b]:cu[b + 1], h * G:(h + 1) * G].double().reshape(new * G, hd)
                s = rows @ k.t() / math.sqrt(hd)
                if new > 1:
                    hidden = torch.ones(new, held, device=DEV).triu(past[b] + 1).bool().repeat_interleave(G, 0)
                    s[:, n:].masked_fill_(hidden, float("-inf"))
                out[cu[b]:cu[b + 1], h * G:(h + 1) * G] = (torch.softmax(s, -1) @ v).view(new, G, hd)
    return out


def _exact_sample(st):
    """Row by row: the value that the last kept token has, and how many of that value."""
    f = st["filters"]
    of = lambda name, r, other: float(f[name][r]) if isinstance(f.get(name), torch.Tensor) else \
        float(torch.tensor(f.get(name, other), dtype=torch.float32))  # noqa: E731
    tokens, logps = [], []
    for r in range(st["logits"].shape[0]):
        z = st["logits"][r].double()
        t, k, p, low = of("temperature", r, 1.0), int(of("top_k", r, 0)), of("top_p", r, 1.0), of("min_p", r, 0.0)
        best = z.max()
        if t <= 0:
            tokens.append(torch.nonzero(z == best)[0, 0].to(torch.int32))
            logps.append(torch.zeros((), dtype=torch.float64, device=DEV))
            continue
        w = torch.exp((z - best) / t)
        down = torch.argsort(z, descending=True, stable=True)
        if 0 < k < len(z):
            w[down[k:]] = 0
        if p < 1:
            sums = torch.cumsum(w[down], 0)
            last = int(torch.searchsorted(sums, p * sums[-1:], right=False)[0])
            w[down[last + 1:]] = 0
        w[w < low] = 0
        sums = torch.cumsum(w, 0)
        token = torch.searchsorted(sums, st["uniform"][r:r + 1].double() * sums[-1], right=True)[0]
        tokens.append(token.to(torch.int32))
        logps.append(torch.log(w[token]) - torch.log(sums[-1]))
    return dict(tokens=torch.stack(tokens), logprobs=torch.stack(logps))


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](st)
