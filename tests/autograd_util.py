"""The two model families' forward pass in float64 torch on the CPU, for gradients of
any loss over the logits by automatic differentiation (tests only; pinned to the
NumPy oracle in test_train_losses_cpu.py)."""
import math

import numpy as np
import torch


def _attention(q, k, v):
    """causal attention of one sequence: q [s, H, hd], k / v [s, KV, hd]"""
    s, H, hd = q.shape
    k, v = (t.repeat_interleave(H // t.shape[1], 1) for t in (k, v))
    a = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(hd)
    a = a.masked_fill(torch.ones(s, s, dtype=torch.bool).triu(1), -math.inf)
    return torch.einsum("hqk,khd->qhd", torch.softmax(a, -1), v).reshape(s, H * hd)


def _gpt2(cfg, w, ids):
    D, H, eps = cfg["hidden_size"], cfg["num_attention_heads"], cfg["layer_norm_epsilon"]
    ln = lambda x, n: torch.nn.functional.layer_norm(x, (D,), w[n + ".weight"], w[n + ".bias"], eps)  # noqa: E731
    lin = lambda x, n: x @ w[n + ".weight"] + w[n + ".bias"]  # noqa: E731
    s = len(ids)
    x = w["transformer.wte.weight"][ids] + w["transformer.wpe.weight"][:s]
    for i in range(cfg["num_hidden_layers"]):
        p = f"transformer.h.{i}."
        q, k, v = (t.reshape(s, H, D // H) for t in lin(ln(x, p + "ln_1"), p + "attn.c_attn").split(D, -1))
        x = x + lin(_attention(q, k, v), p + "attn.c_proj")
        z = lin(ln(x, p + "ln_2"), p + "mlp.c_fc")
        x = x + lin(torch.nn.functional.gelu(z, approximate="tanh"), p + "mlp.c_proj")
    return ln(x, "transformer.ln_f") @ w["transformer.wte.weight"].T


def _llama(cfg, w, ids):
    H, KV, hd, eps = cfg["num_attention_heads"], cfg["num_key_value_heads"], cfg["head_dim"], cfg["rms_norm_eps"]
    norm = lambda x, n: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w[n + ".weight"]  # noqa: E731
    s = len(ids)
    ang = torch.arange(s, dtype=torch.float64)[:, None] * cfg["rope_theta"] ** (
        -2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]

    def rot(t):
        a, b = t[..., :hd // 2], t[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    x = w["model.embed_tokens.weight"][ids]
    for i in range(cfg["num_hidden_layers"]):
        p = f"model.layers.{i}."
        h = norm(x, p + "input_layernorm")
        q, k, v = (h @ w[p + f"self_attn.{n}_proj.weight"].T
                   + (w[p + f"self_attn.{n}_proj.bias"] if cfg["attention_bias"] else 0.0) for n in "qkv")
        o = _attention(rot(q.view(s, H, hd)), rot(k.view(s, KV, hd)), v.view(s, KV, hd))
        x = x + o @ w[p + "self_attn.o_proj.weight"].T
        h = norm(x, p + "post_attention_layernorm")
        a = torch.nn.functional.silu(h @ w[p + "mlp.gate_proj.weight"].T) * (h @ w[p + "mlp.up_proj.weight"].T)
        x = x + a @ w[p + "mlp.down_proj.weight"].T
    head = "model.embed_tokens.weight" if cfg["tie_word_embeddings"] else "lm_head.weight"
    return norm(x, "model.norm") @ w[head].T


def logits(cfg, weights, seqs):
    """[sum of lengths, V] of the packed sequences, each from position 0"""
    f = _gpt2 if cfg.get("model_type") == "gpt2" else _llama
    return torch.cat([f(cfg, weights, torch.as_tensor(np.asarray(s), dtype=torch.long)) for s in seqs])


def loss_and_grads(cfg, weights, seqs, loss):
    """loss(log-probabilities [tokens, V]) and its gradient at every weight (float64)"""
    w = {k: v.detach().cpu().double().requires_grad_() for k, v in weights.items()}
    value = loss(torch.log_softmax(logits(cfg, w, seqs), -1))
    value.backward()
    return float(value.detach()), {k: (v.grad if v.grad is not None else torch.zeros_like(v)).numpy() for k, v in w.items()}


def at_targets(logp, targets):
    """log-probability of each counted target, 0 elsewhere; and which count"""
    tg = torch.as_tensor(np.asarray(targets), dtype=torch.long)
    ok = (tg >= 0) & (tg < logp.shape[1])
    return torch.where(ok, logp[torch.arange(len(tg)), tg.clamp(0, logp.shape[1] - 1)], 0.0), ok


def cross_entropy(targets):
    def loss(logp):
        lp, ok = at_targets(logp, targets)
        return -lp.sum() / ok.sum()
    return loss


def preference(targets, cu, ref, beta, e):
    def loss(logp):
        lp, _ = at_targets(logp, targets)
        s = torch.stack([lp[a:b].sum() for a, b in zip(cu, cu[1:])]) - torch.as_tensor(ref, dtype=torch.float64)
        u = beta * (s[0::2] - s[1::2])
        ls = torch.nn.functional.logsigmoid
        return -((1 - e) * ls(u) + e * ls(-u)).mean()
    return loss


def policy(targets, cu, old, adv, ref, lo, hi, kl, per):
    def loss(logp):
        lp, ok = at_targets(logp, targets)
        o, a, r = (torch.where(ok, torch.as_tensor(v, dtype=torch.float64), 0.0) for v in (old, adv, ref))
        q = torch.exp(lp - o)
        each = -torch.minimum(q * a, q.clamp(1 - lo, 1 + hi) * a) + kl * (torch.exp(r - lp) - (r - lp) - 1)
        each = torch.where(ok, each, 0.0)
        if not per:
            return each.sum() / ok.sum()
        n = [(each[x:y].sum(), int(ok[x:y].sum())) for x, y in zip(cu, cu[1:])]
        return sum(v / c for v, c in n if c) / sum(1 for _, c in n if c)
    return loss
