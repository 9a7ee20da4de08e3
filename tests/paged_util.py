"""Inputs of the paged-cache operators and their plain form in float64."""
import math

import torch

U = 2.0 ** -24
F, B = torch.float32, torch.bfloat16
HALF = {F: U, B: 2.0 ** -8}  # half a step of the type, relative


class Paged:
    """Sequences in groups that share a prefix, their pages in random order.  ``groups``
    lists (prefix length, [(own keys before the call, new tokens), ...])."""

    def __init__(self, groups, heads, kv, hd, dtype, page=16, seed=0, cu=None, junk=True, spare=1):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv, self.hd, self.dtype, self.page = heads, kv, hd, dtype, page
        self.prefix = [n for n, _ in groups]
        self.past = [p for _, s in groups for p, _ in s]
        self.new = [n for _, s in groups for _, n in s]
        self.cu_groups = [0]
        for _, s in groups:
            self.cu_groups.append(self.cu_groups[-1] + len(s))
        self.cu = [0]
        for n in self.new:
            self.cu.append(self.cu[-1] + n)
        self.cu_seqlens = self.cu if (cu or any(n != 1 for n in self.new)) else None
        self.T = self.cu[-1]
        own = [p + n for p, n in zip(self.past, self.new)]
        need = sum(-(-n // page) for n in own + self.prefix)
        self.num_pages = need + spare
        ids = torch.randperm(self.num_pages, generator=g).tolist()

        def table(lens):
            t = torch.full((len(lens), max([1] + [-(-n // page) for n in lens])), -1, dtype=torch.int32)
            for i, n in enumerate(lens):
                for j in range(-(-n // page)):
                    t[i, j] = ids.pop()
            return t.cuda()
        self.table, self.prefix_table = table(own), table(self.prefix)
        self.lens = torch.tensor(self.past, dtype=torch.int32).cuda()
        self.prefix_lens = torch.tensor(self.prefix, dtype=torch.int32).cuda()
        rnd = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
        self.k_cache, self.v_cache = (rnd(self.num_pages, kv, page, hd) for _ in range(2))
        if junk:  # behind the last keys, and in pages of nobody
            used = torch.zeros(self.num_pages, page, dtype=torch.bool)
            for t, lens in ((self.table, own), (self.prefix_table, self.prefix)):
                for i, n in enumerate(lens):
                    for j in range(n):
                        used[int(t[i, j // page]), j % page] = True
            hide = ~used[:, None, :, None]
            self.k_cache = torch.where(hide, torch.tensor(float("nan"), dtype=dtype), self.k_cache)
            self.v_cache = torch.where(hide, torch.tensor(float("-inf"), dtype=dtype), self.v_cache)
        self.k_cache, self.v_cache = self.k_cache.cuda(), self.v_cache.cuda()
        self.q = rnd(self.T, heads, hd).cuda()
        self.k, self.v = rnd(self.T, kv, hd).cuda(), rnd(self.T, kv, hd).cuda()

    def attention_args(self):
        return dict(prefix_table=self.prefix_table, prefix_lens=self.prefix_lens, cu_groups=self.cu_groups,
                    cu_seqlens=self.cu_seqlens)

    def keys(self, cache, table, n, kvh):
        """float64 [n, hd] and whether each key has a page"""
        at = torch.arange(n)
        col = at // self.page
        inside = col < table.shape[0]
        page = torch.where(inside, table.cpu().long()[col.clamp(max=table.shape[0] - 1)], -1)
        ok = (page >= 0) & (page < self.num_pages)
        rows = cache.cpu()[page.clamp(0, self.num_pages - 1), kvh, at % self.page].double()
        return rows, ok

    def attention(self, q=None, scale=None):
        """(out, bound of the error, lse, its bound), float64 on the CPU.

        With u = 2^-24 and h half a step of the type: a score is a float32 sum of hd
        products, off by (hd + 2) u sum |q k| scale = d; a weight exp(s - max) is off by
        d of the score and of the maximum, and by (3 |s - max| + 8) u of itself (base 2,
        its product, the hardware's exponential, at most three rescalings); a bf16 weight
        is rounded (h) before it multiplies v; the n products are added in some order
        (n u).  The sum of the weights is off by the same without h.  So out is off by
        (2 (2 d + (3 x + 8) u + n u) + h) sum p |v| and its own rounding h |out|."""
        q = (self.q if q is None else q).cpu().double()
        scale = self.hd ** -0.5 if scale is None else scale
        G = self.heads // self.kv
        out = torch.zeros(q.shape, dtype=torch.float64)
        bound, lse, lse_bound = torch.zeros_like(out), torch.full(out.shape[:2], -math.inf, dtype=torch.float64), None
        lse_bound = torch.zeros_like(lse)
        h = 0.0 if self.dtype == F else HALF[B]
        for b in range(len(self.past)):
            past = int(self.lens[b])
            if past < 0:
                continue
            group = [g for g in range(len(self.prefix)) if self.cu_groups[g] <= b < self.cu_groups[g + 1]]
            new = self.cu[b + 1] - self.cu[b]
            for kvh in range(self.kv):
                parts = [self.keys(c, self.prefix_table[g], max(0, int(self.prefix_lens[g])), kvh) for g in group
                         for c in (self.k_cache, self.v_cache)]
                own = [self.keys(c, self.table[b], past + new, kvh) for c in (self.k_cache, self.v_cache)]
                for i in range(new):
                    n = past + i + 1
                    k = torch.cat([p[0] for p in parts[0::2]] + [own[0][0][:n]])
                    v = torch.cat([p[0] for p in parts[1::2]] + [own[1][0][:n]])
                    ok = torch.cat([p[1] for p in parts[0::2]] + [own[0][1][:n]])
                    k, v = k[ok], v[ok]
                    if len(k) == 0:
                        continue
                    for h_ in range(kvh * G, (kvh + 1) * G):
                        row = q[self.cu[b] + i, h_]
                        s = (k @ row) * scale
                        d = (self.hd + 2) * U * (k.abs() @ row.abs()) * abs(scale)
                        x = s.max() - s
                        p = torch.softmax(s, 0)
                        eps = 2 * d.max() + (p * (3 * x + 8)).max() * U + 8 * U + len(k) * U
                        o, a = p @ v, p @ v.abs()
                        at = (self.cu[b] + i, h_)
                        out[at], lse[at] = o, torch.logsumexp(s, 0)
                        bound[at] = (2 * eps + h) * a + HALF[self.dtype] * (o.abs() + (2 * eps + h) * a)
                        lse_bound[at] = eps + 4 * U * (1 + lse[at].abs() + s.abs().max())
        return out, bound + 1e-38, lse, lse_bound


def check(got, ref, bound, what):
    got = got.detach().cpu().double()
    off = (got - ref).abs()
    off = torch.where(got == ref, 0.0, off)  # (infinities)
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((off / bound.clamp_min(1e-300)).max()))
