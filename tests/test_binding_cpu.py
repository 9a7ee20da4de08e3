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
