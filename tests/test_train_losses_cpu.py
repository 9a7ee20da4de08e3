"""Pins of the float64 torch models against the NumPy oracle, and the refusals of the
training step's losses, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import autograd_util as ag
import oracle
from paper_2608_19889_amd import axon as ax
from synthetic import model_weights, prompts, small_shape
from test_gpu_gpt2 import gpt2_shape


def _seqs(lens, vocab, seed):
    ids = prompts(len(lens), max(lens), vocab, seed=seed).numpy()
    return [ids[i, :n] for i, n in enumerate(lens)]


@pytest.mark.parametrize("base,ov", [("1b", dict(hidden=128, intermediate=192)), ("7b", dict(hidden=128, intermediate=64))])
def test_llama_gradients_equal_the_oracles(base, ov):
    shape = small_shape(base, layers=2, vocab=90, **ov)
    w, seqs = model_weights(shape, seed=1), _seqs([9, 1, 14], 90, 2)
    tg = [np.append(s[1:], -1) for s in seqs]
    loss, grads = oracle.loss_and_grads(shape, oracle.weights_f64(w), seqs, tg)
    mine, got = ag.loss_and_grads(shape, w, seqs, ag.cross_entropy(np.concatenate(tg)))
    assert abs(loss - mine) < 1e-12
    for k, v in grads.items():
        np.testing.assert_allclose(got[k], v, atol=1e-12, err_msg=k)


def test_gpt2_logits_equal_the_oracles():
    shape = gpt2_shape(hidden=128, heads=2, vocab=90, positions=32)
    w, seqs = model_weights(shape, seed=3), _seqs([9, 1, 14], 90, 4)
    want = oracle.OracleDecoder(shape, w).prefill(seqs, all_logits=True)
    got = ag.logits(shape, {k: v.double() for k, v in w.items()}, seqs).numpy()
    np.testing.assert_allclose(got, np.concatenate(list(want)), atol=1e-11)


def test_refusals_of_the_training_losses():
    """Checked on the host before the model is touched."""
    L = ax.lib()
    cu = (ctypes.c_int32 * 3)(0, 2, 4)
    P = 1 << 20
    for change, text in [(dict(m=None), "model is NULL")]:
        rc = L.axon_preference_loss_and_grads(None, 1, P, P, cu, P, None, 0.1, 0.0, P, P, P, None, 0, None)
        assert rc == ax.AXON_E_INVALID and text in ax.last_error()
        rc = L.axon_policy_loss_and_grads(None, 1, P, P, cu, P, P, None, P, 0.2, 0.2, 0.0, 0, P, P, P, None, 0, None)
        assert rc == ax.AXON_E_INVALID and text in ax.last_error()


class NoModel:
    _h = None
    _train_args = ax.Model._train_args


def test_binding_refuses_what_a_step_cannot_take():
    """Host tensors and mixed devices never reach the library as pointers."""
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="on the GPU"):
        ax.Model.policy_loss_and_grads(NoModel(), i, [0, 2, 4], i, {"w": f}, f, f)
    with pytest.raises(ValueError, match="on the GPU"):
        ax.Model.preference_loss_and_grads(NoModel(), i, [0, 2, 4], i, {"w": f})
    meta = torch.zeros(4, dtype=torch.int32, device="meta")
    with pytest.raises(ValueError, match="on the GPU"):
        ax.Model.preference_loss_and_grads(NoModel(), meta, [0, 2, 4], i, {"w": f})
    for tokens, targets, grads, text in [(i.long(), i, {}, "tokens must hold 4"), (i, i[:3], {}, "targets must hold 4"),
                                         (i, i, {"w": torch.zeros(3, 2).t()}, "buffer of w is not contiguous")]:
        with pytest.raises(ValueError, match=text):
            NoModel()._train_args(tokens, [0, 2, 4], targets, grads)
