"""Refusals of the preference and policy steps that need no model: they are checked on
the host before the model (a number that is never followed here) is read."""
import ctypes

import pytest

from paper_2608_19889_amd import axon as ax

P = 1 << 20
CU = (ctypes.c_int32 * 3)(0, 2, 4)
NAN, INF = float("nan"), float("inf")
PREF = dict(m=P, pairs=1, tokens=P, d_cu=P, h_cu=CU, targets=P, ref=None, beta=0.1, e=0.0, loss=P, seq=P, margins=P,
            grads=None, n=0, stream=None)
POL = dict(m=P, batch=2, tokens=P, d_cu=P, h_cu=CU, targets=P, old=P, ref=None, adv=P, lo=0.2, hi=0.2, kl=0.0, per=0,
           loss=P, stats=P, logps=P, grads=None, n=0, stream=None)
CALLS = {"preference": PREF, "policy": POL}
BAD = [
    ("preference", dict(m=None), "model is NULL"),
    ("preference", dict(pairs=0), "pairs"),
    ("preference", dict(pairs=(1 << 29) + 1), "pairs"),
    ("preference", dict(beta=0.0), "beta"),
    ("preference", dict(beta=NAN), "beta"),
    ("preference", dict(beta=INF), "beta"),
    ("preference", dict(e=-0.1), "label_smoothing"),
    ("preference", dict(e=0.5), "label_smoothing"),
    ("preference", dict(e=NAN), "label_smoothing"),
    ("preference", dict(seq=None), "d_seq_logps"),
    ("preference", dict(margins=None), "d_margins"),
    ("policy", dict(m=None), "model is NULL"),
    ("policy", dict(lo=-0.1), "clip_low"),
    ("policy", dict(lo=1.1), "clip_low"),
    ("policy", dict(hi=-0.1), "clip_high"),
    ("policy", dict(hi=INF), "clip_high"),
    ("policy", dict(kl=-1.0), "kl_coef"),
    ("policy", dict(kl=NAN), "kl_coef"),
    ("policy", dict(kl=0.1), "needs d_ref_logps"),
    ("policy", dict(per=2), "per_sequence"),
    ("policy", dict(old=None), "d_old_logps"),
    ("policy", dict(adv=None), "d_advantages"),
    ("policy", dict(stats=None), "d_stats"),
    ("policy", dict(logps=None), "d_logps"),
]


@pytest.mark.parametrize("step,change,text", BAD, ids=["%s-%s-%s" % (b[0], *b[1], *b[1].values()) for b in BAD])
def test_refusals(step, change, text):
    rc = getattr(ax.lib(), f"axon_{step}_loss_and_grads")(*{**CALLS[step], **change}.values())
    assert rc == ax.AXON_E_INVALID and text in ax.last_error()
