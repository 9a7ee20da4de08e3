"""The Python binding on the GPU: devices of a model and of its arguments, buffers that
autograd holds."""
import pytest
import torch

import paper_2608_19889_amd as ops
from test_gpu_train_losses import FAMILIES, setup

pytestmark = pytest.mark.gpu


def test_a_buffer_that_autograd_holds():
    x = torch.randn(6, 50, device="cuda", requires_grad=True)
    tg = torch.zeros(6, dtype=torch.int32, device="cuda")
    g = torch.ones(50, device="cuda")
    for call in (lambda y: ops.layernorm(y, g, out=y), lambda y: ops.layernorm_backward(x.detach(), y, g, dx=y),
                 lambda y: ops.token_logprobs_backward(y, tg, tg.float(), dlogits=y),
                 lambda y: ops.preference_loss(y, tg, [0, 2, 6], dlogits=y),
                 lambda y: ops.policy_loss(y, tg, [0, 6], tg.float(), tg.float(), dlogits=y)):
        y = x.exp()  # (its backward pass needs y)
        call(y.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_a_step_on_another_device_than_the_models_is_refused():
    """Its weights and work buffers lie on the device that was current when it was made."""
    shape, lens = FAMILIES["gpt2"]
    w, seqs, tg, m, flat, cu, targets, grads = setup(shape, lens, 111)
    f = torch.zeros(len(tg), device="cuda")
    assert m.device == torch.device("cuda", torch.cuda.current_device())
    m.device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="tensors on cuda:0, the model on cuda:1"):
        m.policy_loss_and_grads(flat, cu, targets, grads, f, f)
    with pytest.raises(ValueError, match="tensors on cuda:0, the model on cuda:1"):
        m.preference_loss_and_grads(flat, cu, targets, grads)
    m.close()
