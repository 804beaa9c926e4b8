"""Entries of the table and logits that are infinite."""
import pytest

from test_vocab_gpu import DEV, Ends

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slots", [20, 100, 300])
def test_an_infinite_entry_of_the_target(slots):
    """A target whose logit is -inf: the gradient of that column is infinite, not undefined, and the row's others are finite."""
    import torch
    e = Ends(25, [slots + 1], 1, 0, 300, 64, masked=0.0)
    e.tok[:] = 7
    e.target[:-1] = 7
    e.tokens.fill_(7)
    e.table[7, 5] = float("inf")
    e.x = torch.randn(slots + 1, 64, device=DEV).bfloat16()
    e.x[:, 5] = -e.x[:, 5].abs() - 0.125
    e.d_loss = torch.rand(slots + 1, device=DEV) + 0.1
    loss, lse = e.loss()
    assert (loss[:-1] == float("inf")).all() and torch.isfinite(lse[:-1]).all()
    dx, _ = e.loss_bwd(lse)
    assert torch.isneginf(dx[:-1, 5]).all()
    dx[:, 5] = 0
    assert torch.isfinite(dx).all()
