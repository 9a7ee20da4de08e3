"""What the Python binding does with its arguments before the library sees them, without a
GPU."""
import pytest
import torch

from paper_2608_19889_amd import axon as ax


class NoModel:
    _h = None
    _train_args = ax.Model._train_args


@pytest.mark.parametrize("first", ["grads", "cu_seqlens", "tokens"])
def test_keyword_arguments_of_a_step_come_in_any_order(first):
    """What decides is where the tensors lie, not which argument is written first."""
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    kw = dict(tokens=i, cu_seqlens=[0, 2, 4], targets=i, grads={"w": f})
    kw = {first: kw.pop(first), **kw}
    with pytest.raises(ValueError, match="takes tensors on the GPU, got one on cpu"):
        ax.Model.preference_loss_and_grads(NoModel(), **kw)
    with pytest.raises(ValueError, match="takes tensors on the GPU, got one on cpu"):
        ax.Model.policy_loss_and_grads(NoModel(), old_logps=f, advantages=f, **kw)


def test_a_callers_buffer_counts_as_modified():
    """Autograd cannot see a write through a pointer: the buffer's version says so, and a
    backward pass that needs what stood there is refused, not wrong."""
    x = torch.randn(4, 3, requires_grad=True)
    y = (x * 2).exp()
    before = y._version
    assert ax._like(y.detach(), x, torch.float32, "out") is not None
    assert y._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    # a refused buffer, and a new one, leave everything as it was
    z = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="out must be"):
        ax._like(z, x, torch.float32, "out")
    ax._like(None, x, torch.float32, "out")
    assert z._version == 0 and x._version == 0


def test_docstrings_say_that_autograd_sees_nothing():
    for f in (ax.layernorm, ax.layernorm_backward, ax.token_logprobs, ax.token_logprobs_backward, ax.preference_loss,
              ax.policy_loss, ax.Model.preference_loss_and_grads, ax.Model.policy_loss_and_grads):
        assert "autograd" in f.__doc__ and "``stream``" in f.__doc__
