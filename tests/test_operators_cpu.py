"""Refusals of the row operators: every check runs on the host before any HIP call,
so these need no GPU (the pointers are numbers that are never followed)."""
import ctypes

import pytest
import torch

import paper_2608_19889_amd as ops
from paper_2608_19889_amd import axon as ax

P = 1 << 20  # a "device pointer"
F, B = ax.AXON_F32, ax.AXON_BF16
BIG = 1 << 40


def cu(*v):
    return (ctypes.c_int32 * len(v))(*v)


LN = dict(rows=4, cols=64, x=P, x_dtype=F, ldx=64, gain=P, bias=P, param_dtype=F, eps=1e-5, y=2 * P, y_dtype=F, ldy=64,
          stream=None)
LNB = dict(rows=4, cols=64, x=P, x_dtype=F, ldx=64, dy=2 * P, dy_dtype=F, lddy=64, gain=P, param_dtype=F, eps=1e-5,
           dx=3 * P, lddx=64, dgain=P, dbias=P, ws=P, ws_bytes=BIG, stream=None)
ROWS = dict(tokens=6, vocab=50, z=P, dtype=F, ld=50, targets=P)
GRAD = dict(dz=2 * P, gdtype=F, ldg=50)
WORK = dict(ws=P, ws_bytes=BIG, stream=None)
LP = dict(ROWS, logps=P, **WORK)
LPB = dict(ROWS, dlogps=P, **GRAD, stream=None)
PREF = dict(ROWS, pairs=1, d_cu=P, h_cu=cu(0, 2, 6), ref=P, beta=0.1, e=0.1, loss=P, seq=P, margins=P, **GRAD, **WORK)
POL = dict(ROWS, batch=2, d_cu=P, h_cu=cu(0, 2, 6), old=P, ref=P, adv=P, lo=0.2, hi=0.2, kl=0.1, per=0, loss=P, stats=P,
           logps=P, **GRAD, **WORK)
CALLS = {"axon_layernorm": LN, "axon_layernorm_backward": LNB, "axon_token_logprobs": LP,
         "axon_token_logprobs_backward": LPB, "axon_preference_loss": PREF, "axon_policy_loss": POL}

NAN, INF = float("nan"), float("inf")
BAD = [
    ("axon_layernorm", dict(rows=-1), ax.AXON_E_INVALID, "rows"),
    ("axon_layernorm", dict(cols=0), ax.AXON_E_INVALID, "cols"),
    ("axon_layernorm", dict(cols=16385, ldx=20000, ldy=20000), ax.AXON_E_INVALID, "cols"),
    ("axon_layernorm", dict(eps=0.0), ax.AXON_E_INVALID, "eps"),
    ("axon_layernorm", dict(eps=NAN), ax.AXON_E_INVALID, "eps"),
    ("axon_layernorm", dict(ldx=63), ax.AXON_E_INVALID, "stride of x"),
    ("axon_layernorm", dict(ldy=63), ax.AXON_E_INVALID, "stride of y"),
    ("axon_layernorm", dict(x=None), ax.AXON_E_INVALID, "x is NULL"),
    ("axon_layernorm", dict(x=P + 2), ax.AXON_E_INVALID, "aligned"),
    ("axon_layernorm", dict(x_dtype=3), ax.AXON_E_DTYPE, "x must be"),
    ("axon_layernorm", dict(y_dtype=0), ax.AXON_E_DTYPE, "y must be"),
    ("axon_layernorm", dict(param_dtype=7), ax.AXON_E_DTYPE, "gain"),
    ("axon_layernorm", dict(gain=None), ax.AXON_E_INVALID, "gain"),
    ("axon_layernorm", dict(y=P, y_dtype=B), ax.AXON_E_INVALID, "x's buffer"),
    ("axon_layernorm", dict(y=P, ldy=70), ax.AXON_E_INVALID, "x's buffer"),
    ("axon_layernorm_backward", dict(dgain=None), ax.AXON_E_INVALID, "dgain"),
    ("axon_layernorm_backward", dict(ws_bytes=100), ax.AXON_E_CAPACITY, "workspace"),
    ("axon_layernorm_backward", dict(ws=None), ax.AXON_E_INVALID, "workspace"),
    ("axon_layernorm_backward", dict(ws=P + 4), ax.AXON_E_INVALID, "16 bytes"),
    ("axon_layernorm_backward", dict(lddx=60), ax.AXON_E_INVALID, "stride of dx"),
    ("axon_layernorm_backward", dict(dx=2 * P, dy_dtype=B), ax.AXON_E_INVALID, "buffer of x or dy"),
    ("axon_layernorm_backward", dict(dx=P, lddx=80), ax.AXON_E_INVALID, "buffer of x or dy"),
    ("axon_token_logprobs", dict(tokens=-1), ax.AXON_E_INVALID, "tokens"),
    ("axon_token_logprobs", dict(vocab=0), ax.AXON_E_INVALID, "vocab"),
    ("axon_token_logprobs", dict(ld=49), ax.AXON_E_INVALID, "stride of logits"),
    ("axon_token_logprobs", dict(dtype=9), ax.AXON_E_DTYPE, "logits"),
    ("axon_token_logprobs", dict(targets=None), ax.AXON_E_INVALID, "d_targets"),
    ("axon_token_logprobs", dict(logps=None), ax.AXON_E_INVALID, "d_logps"),
    ("axon_token_logprobs", dict(ws_bytes=0), ax.AXON_E_CAPACITY, "workspace"),
    ("axon_token_logprobs_backward", dict(dz=None), ax.AXON_E_INVALID, "dlogits"),
    ("axon_token_logprobs_backward", dict(dz=P, gdtype=B), ax.AXON_E_INVALID, "logits' buffer"),
    ("axon_token_logprobs_backward", dict(dz=P, ldg=64), ax.AXON_E_INVALID, "logits' buffer"),
    ("axon_token_logprobs_backward", dict(ldg=10), ax.AXON_E_INVALID, "stride of dlogits"),
    ("axon_token_logprobs_backward", dict(dlogps=None), ax.AXON_E_INVALID, "d_dlogps"),
    ("axon_preference_loss", dict(pairs=0), ax.AXON_E_INVALID, "pairs"),
    ("axon_preference_loss", dict(beta=0.0), ax.AXON_E_INVALID, "beta"),
    ("axon_preference_loss", dict(beta=INF), ax.AXON_E_INVALID, "beta"),
    ("axon_preference_loss", dict(e=0.5), ax.AXON_E_INVALID, "label_smoothing"),
    ("axon_preference_loss", dict(e=-0.1), ax.AXON_E_INVALID, "label_smoothing"),
    ("axon_preference_loss", dict(h_cu=cu(1, 2, 6)), ax.AXON_E_INVALID, r"cu_seqlens\[0\]"),
    ("axon_preference_loss", dict(h_cu=cu(0, 7, 6)), ax.AXON_E_INVALID, "length -1"),
    ("axon_preference_loss", dict(h_cu=cu(0, 2, 5)), ax.AXON_E_INVALID, "end at 5"),
    ("axon_preference_loss", dict(h_cu=None), ax.AXON_E_INVALID, "h_cu_seqlens"),
    ("axon_preference_loss", dict(d_cu=None), ax.AXON_E_INVALID, "d_cu_seqlens"),
    ("axon_preference_loss", dict(margins=None), ax.AXON_E_INVALID, "d_margins"),
    ("axon_preference_loss", dict(gdtype=5), ax.AXON_E_DTYPE, "dlogits"),
    ("axon_policy_loss", dict(batch=0), ax.AXON_E_INVALID, "batch"),
    ("axon_policy_loss", dict(lo=1.5), ax.AXON_E_INVALID, "clip_low"),
    ("axon_policy_loss", dict(lo=NAN), ax.AXON_E_INVALID, "clip_low"),
    ("axon_policy_loss", dict(hi=-0.1), ax.AXON_E_INVALID, "clip_high"),
    ("axon_policy_loss", dict(hi=INF), ax.AXON_E_INVALID, "clip_high"),
    ("axon_policy_loss", dict(kl=-1.0), ax.AXON_E_INVALID, "kl_coef"),
    ("axon_policy_loss", dict(ref=None), ax.AXON_E_INVALID, "d_ref_logps"),
    ("axon_policy_loss", dict(per=2), ax.AXON_E_INVALID, "per_sequence"),
    ("axon_policy_loss", dict(old=None), ax.AXON_E_INVALID, "d_old_logps"),
    ("axon_policy_loss", dict(adv=P + 1), ax.AXON_E_INVALID, "d_advantages"),
    ("axon_policy_loss", dict(stats=None), ax.AXON_E_INVALID, "d_stats"),
]


@pytest.mark.parametrize("call,change,code,text", BAD, ids=["%s-%s" % (b[0][5:], "-".join(b[1])) for b in BAD])
def test_refusals(call, change, code, text):
    with pytest.raises(ax.AxonError, match=text) as e:
        ax._check(getattr(ax.lib(), call)(*{**CALLS[call], **change}.values()))
    assert e.value.code == code


def test_workspaces_grow_with_the_call_and_are_zero_for_what_is_refused():
    L = ax.lib()
    assert L.axon_layernorm_backward_workspace(0, 64) == 0
    assert L.axon_layernorm_backward_workspace(100, 64) > 0
    assert L.axon_layernorm_backward_workspace(5, 1 << 20) == 0
    assert L.axon_token_loss_workspace(-1, 50, 0) == 0
    assert 0 < L.axon_token_loss_workspace(8, 50, 2) < L.axon_token_loss_workspace(4096, 50257, 16)
    # past 32 bits of bytes
    assert L.axon_token_loss_workspace(1 << 29, 50257, 2) > 1 << 33


def test_binding_refuses_what_it_cannot_hand_over():
    x = torch.zeros(4, 8)
    for call in (lambda: ops.layernorm(x, torch.ones(8)), lambda: ops.token_logprobs(x, x[0]),
                 lambda: ops.layernorm_backward(x, x, gain=x[0]),
                 lambda: ops.policy_loss(x, x[0], [0, 4], x[0], x[0], stream=0)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
