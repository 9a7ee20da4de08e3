"""Answers to prompts as a policy step samples them: rotation and append, attention over
prompts that answers share and the draw of a token, run together, and the losses that
learn from what they gave."""
import numpy as np
import pytest
import torch

import paper_2608_19889_amd as ops
from paged_util import B, F, HALF, U, Paged, check
from parity_util import gpu_model, pack
from synthetic import model_weights, prompts, small_shape
from test_gpu_losses import Rows
from test_gpu_paged import rotated
from test_gpu_sample import reference

pytestmark = pytest.mark.gpu
HEADS, KV, HD, STEPS = 4, 2, 64, 21
VOCAB = HEADS * HD  # an attention's output is the next logits
SETTINGS = dict(temperature=0.2, top_k=50, top_p=0.97)


class Decoder:
    """Five answers to two prompts by a model whose layers are one attention."""

    def __init__(self, dtype, seed):
        self.p = p = Paged([(37, [(STEPS - 1, 1)] * 3), (20, [(STEPS - 1, 1)] * 2)], HEADS, KV, HD, dtype, seed=seed)
        g = torch.Generator().manual_seed(seed + 1)
        self.q, self.k, self.v = (torch.randn((VOCAB, h, HD), generator=g).to(dtype).cuda() for h in (HEADS, KV, KV))
        self.uniform = torch.rand((STEPS + 1, 5), generator=g).cuda()
        self.prompt = torch.randint(0, VOCAB, (57,), generator=g).cuda()
        self.inv = 1e4 ** (-torch.arange(0, HD, 2, dtype=torch.float64) / HD).cuda()
        self.offsets = torch.tensor([37] * 3 + [20] * 2, dtype=torch.int32).cuda()
        self.groups = torch.tensor(p.cu_groups, dtype=torch.int32).cuda()
        self.caches = p.k_cache.clone(), p.v_cache.clone()
        self.tokens = torch.zeros((5,), dtype=torch.int32, device="cuda")
        self.u = torch.zeros((5,), device="cuda")

    def start(self):
        """The prompts' keys into the pages of the prefixes; the first tokens."""
        p = self.p
        for cache, kept in zip((p.k_cache, p.v_cache), self.caches):
            cache.copy_(kept)
        p.lens.zero_()
        none = torch.zeros((2,), dtype=torch.int32, device="cuda")
        t = self.prompt
        q = ops.rope_append(self.q[t], self.k[t], self.v[t], p.k_cache, p.v_cache, p.prefix_table, none, self.inv,
                            cu_seqlens=[0, 37, 57])
        out = ops.prefix_attention(q, p.k_cache, p.v_cache, p.prefix_table, none, cu_seqlens=[0, 37, 57])
        z = torch.cat([out[36:37].expand(3, -1, -1), out[56:57].expand(2, -1, -1)]).reshape(5, VOCAB)
        ops.sample_tokens(z, self.uniform[0], out=self.tokens, **SETTINGS)
        self.u.copy_(self.uniform[1])

    def step(self):
        p, t = self.p, self.tokens.long()
        r = ops.rope_append(self.q[t], self.k[t], self.v[t], p.k_cache, p.v_cache, p.table, p.lens, self.inv,
                            offsets=self.offsets)
        out = ops.prefix_attention(r, p.k_cache, p.v_cache, p.table, p.lens, prefix_table=p.prefix_table,
                                   prefix_lens=p.prefix_lens, cu_groups=p.cu_groups, groups_device=self.groups)
        _, lp = ops.sample_tokens(out.view(5, VOCAB), self.u, out=self.tokens, **SETTINGS)
        p.lens.add_(1)
        return r, out, lp

    def answers(self, step):
        """(tokens, log-probabilities, outputs) of every step"""
        self.start()
        got = []
        for i in range(STEPS):
            _, out, lp = step()
            got.append((self.tokens.clone(), lp.clone(), out.clone()))
            self.u.copy_(self.uniform[min(i + 2, STEPS)])
        return got


@pytest.mark.parametrize("dtype", [F, B])
def test_decode_loop_of_groups(dtype):
    """Every step against float64: rotation (bounds of test_append), attention over what
    the cache then holds (Paged.attention) and the token."""
    d = Decoder(dtype, 5)
    d.start()
    p, half, places = d.p, HALF[dtype], torch.arange(37)
    where = [(d.prompt[:37], 0, places), (d.prompt[37:], 1, places[:20])]
    for t, i, pos in where:
        pages = p.prefix_table[i].cpu().long()[pos // 16]
        want, size = rotated(d.k[t], pos, d.inv, HD, False, 1.0)
        check(p.k_cache.cpu()[pages, :, pos % 16], want, 10 * U * size * (1 + half) + half * want.abs(), "prompt")
        assert torch.equal(p.v_cache.cpu()[pages, :, pos % 16], d.v[t].cpu())
    seen = set()
    for i in range(STEPS):
        fed, lens = d.tokens.clone(), p.lens.clone()
        r, out, lp = d.step()
        pos = lens.cpu() + d.offsets.cpu()
        page = p.table.cpu().long()[torch.arange(5), lens.cpu().long() // 16]
        for got, table in ((r, d.q), (p.k_cache.cpu()[page, :, i % 16], d.k)):
            want, size = rotated(table[fed.long()], pos, d.inv, HD, False, 1.0)
            check(got, want, 10 * U * size * (1 + half) + half * want.abs(), ("rotated", i))
        assert torch.equal(p.v_cache.cpu()[page, :, i % 16], d.v[fed.long()].cpu())
        p.q = r
        p.lens.copy_(lens)
        want, bound, _, _ = p.attention()
        check(out, want, bound, ("attention", i))
        p.lens.add_(1)
        z = out.view(5, VOCAB).float().cpu().numpy()
        for b in range(5):
            token, logp = reference(z[b], float(d.u[b]), SETTINGS["temperature"], SETTINGS["top_k"], SETTINGS["top_p"])
            assert int(d.tokens[b]) == token and abs(float(lp[b]) - logp) <= U * abs(logp) + 1e-9, (i, b)
            seen.add(token)
        d.u.copy_(d.uniform[min(i + 2, STEPS)])
    assert len(seen) > 20  # (the answers differ)


def test_two_captured_decode_loops_in_turn():
    """Two graphs, each a step of its own answers, replayed in turn beside eager steps."""
    loops = [Decoder(F, 7), Decoder(B, 8)]
    want = [d.answers(d.step) for d in loops]
    graphs, outs = [], []
    for d in loops:
        d.start()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            d.step()
        torch.cuda.current_stream().wait_stream(side)
        d.start()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(d.step())
        graphs.append(g)
    for d in loops:
        d.start()
    other = Decoder(F, 9)
    other.start()
    for i in range(STEPS):
        for j, d in enumerate(loops):
            graphs[j].replay()
            if i < STEPS - 1:
                other.step()
                other.p.lens.sub_(1)
            tokens, lp, out = want[j][i]
            assert torch.equal(d.tokens, tokens) and torch.equal(outs[j][2], lp) and torch.equal(outs[j][1], out), (i, j)
            d.u.copy_(d.uniform[min(i + 2, STEPS)])


def test_two_loops_on_two_streams_at_once():
    loops = [Decoder(B, 11), Decoder(B, 12)]
    want = [d.answers(d.step) for d in loops]
    streams = [torch.cuda.Stream() for _ in loops]
    got = [[], []]
    for d in loops:
        d.start()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(STEPS):
        for j, d in enumerate(loops):
            with torch.cuda.stream(streams[j]):
                _, out, lp = d.step()
                got[j].append((d.tokens.clone(), lp, out))
                d.u.copy_(d.uniform[min(i + 2, STEPS)])
    torch.cuda.synchronize()
    for j in range(2):
        for i in range(STEPS):
            assert all(torch.equal(a, b) for a, b in zip(got[j][i], want[j][i])), (i, j)


def test_sampling_from_a_model_and_its_policy_loss():
    """Tokens drawn from a model's logits, prompt and decode steps; the log-probabilities
    that were drawn from are the old ones of the policy loss over the same answers."""
    shape = small_shape("135m", layers=2, vocab=1000, dtype="f32")
    w = model_weights(shape, seed=3)
    ids = prompts(3, 12, 1000, seed=4).numpy()
    seqs, steps = [ids[0, :12], ids[1, :5], ids[2, :9]], 6
    m = gpu_model(shape, w, max_batch=3, max_seq=32)
    u = torch.rand((steps, 3), generator=torch.Generator().manual_seed(6)).cuda()
    flat, cu = pack(seqs)
    z, greedy = m.prefill(flat, cu)
    tokens, lps, rows = [], [], []
    for i in range(steps):
        t, lp = ops.sample_tokens(z, u[i])
        cold, zero = ops.sample_tokens(z, u[i], temperature=0.0)
        assert torch.equal(cold, greedy) and not zero.any()
        for b in range(3):
            assert int(t[b]) == reference(z[b].cpu().numpy(), float(u[i, b]))[0]
        tokens.append(t)
        lps.append(lp)
        rows.append(z)
        if i + 1 < steps:
            z = torch.empty((3, 1000), device="cuda")
            _, greedy = m.decode_step(t, logits=z)
    m.close()
    # answer by answer, as the losses take them
    z, t, lp = (torch.stack(x, 1).flatten(0, 1) for x in (rows, tokens, lps))
    r = Rows(z, t)
    want, bound = r.lp.cpu(), (r.E * U + U * r.lp.abs()).cpu()
    check(lp, want, U * want.abs() + 1e-9, "drawn under")
    check(ops.token_logprobs(z, t), want, bound, "token_logprobs")
    adv = torch.randn((3 * steps,), generator=torch.Generator().manual_seed(7)).cuda()
    loss, _, logps, grad = ops.policy_loss(z, t, [0, steps, 2 * steps, 3 * steps], lp, adv)
    check(logps, want, bound, "policy logps")
    # every ratio is 1 but for the two logarithms' errors and four roundings
    off = (torch.expm1(bound + U * want.abs() + 1e-9) + 4 * U) * adv.double().abs().cpu()
    n = 3 * steps
    assert abs(float(loss) + float(adv.double().mean())) <= float(off.mean()) + (n + 2) * U * float(adv.double().abs().mean())
    assert torch.isfinite(grad).all() and grad.shape == z.shape
