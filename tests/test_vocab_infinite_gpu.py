"""Entries of the table and logits that are infinite, as the definition has them: lse = ln(sum of exponentials), loss = lse - l[target]."""
import numpy as np
import pytest

import vocab_plain as plain
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


@pytest.mark.parametrize("slots,vocab,hidden", [(20, 1000, 64), (60, 70001, 136), (120, 777, 1032), (300, 2000, 64), (300, 700, 1544), (2500, 3000, 200)])
def test_logits_beyond_the_largest_float(slots, vocab, hidden):
    """Two words (one of them in the last, partial tile) have a column that takes the logits of some slots to +inf, of others to -inf."""
    import torch
    e = Ends(31, [slots], 1, 0, vocab, hidden, masked=0.0)
    far = [3, vocab - 1]
    others = [v for v in range(vocab) if v not in far]
    up, down = np.arange(slots) % 5 == 1, np.arange(slots) % 5 == 3
    e.tok = np.random.default_rng(1).choice(others, size=slots).astype(np.int32)
    e.tok[2::7] = far[0]
    e.tok[5::9] = far[1]
    e.tokens = torch.from_numpy(e.tok).to(DEV)
    e.target = plain.targets(e.tok, e.q_idx, e.cu, vocab)
    e.table[:, 0] = 0
    e.table[far, 0] = 1e30
    e.x = torch.randn(slots, hidden, device=DEV, generator=torch.Generator(DEV).manual_seed(2)).bfloat16()
    e.x[:, 0] = torch.from_numpy(np.where(up, 1e30, np.where(down, -1e30, 0.0))).to(DEV)
    e.d_loss = torch.rand(slots, device=DEV)
    has, is_far = e.target >= 0, np.isin(e.target, far)
    dev = lambda m: torch.from_numpy(m).to(DEV)  # noqa: E731
    loss, lse = e.loss()
    inf = torch.tensor(float("inf"), device=DEV)
    assert (lse[dev(up & has)] == inf).all()
    assert (loss[dev(up & has & ~is_far)] == inf).all() and torch.isnan(loss[dev(up & has & is_far)]).all()
    # -inf: such a word adds nothing; as a target it is infinitely unlikely
    place = np.full(vocab, -1)
    place[others] = np.arange(len(others))
    target = np.where(has & down, np.where(is_far, 0, place[np.maximum(e.target, 0)]), -1)
    want = plain.loss(e.x, e.table[others], target, 1.0)
    rows = dev(has & down)
    plain.check("lse", lse[rows], want[1][rows], want[3][rows])
    rows = dev(has & down & ~is_far)
    plain.check("loss", loss[rows], want[0][rows], want[2][rows])
    assert (loss[dev(has & down & is_far)] == inf).all()
    rows = dev(has & ~up & ~down)
    want = plain.loss(e.x[rows], e.table, e.target[has & ~up & ~down], 1.0)
    plain.check("lse", lse[rows], want[1], want[3])
    plain.check("loss", loss[rows], want[0], want[2])
    dx, dt = e.loss_bwd(lse)
    assert torch.isfinite(dx[dev(~up)]).all() and torch.isfinite(dt[others]).all()
    assert torch.isnan(dx[dev(up & has)]).all() and torch.isnan(dt[far]).all()


@pytest.mark.parametrize("slots,vocab,hidden", [(20, 300, 64), (25, 70001, 136), (200, 1000, 64), (1500, 777, 1032)])
def test_an_infinite_gradient_of_one_loss(slots, vocab, hidden):
    """Few slots with a target, one of them with an infinite weight: the table's gradient is infinite with the sign that the definition gives, not undefined."""
    import torch
    e = Ends(32, [slots], 1, 0, vocab, hidden, masked=0.0, logit=1.0)
    tok = np.full(slots, -1, np.int32)
    tok[1:18] = np.random.default_rng(4).integers(0, vocab, 17)
    e.tok, e.tokens = tok, torch.from_numpy(tok).to(DEV)
    e.target = plain.targets(tok, e.q_idx, e.cu, vocab)
    e.x = torch.randn(slots, hidden, device=DEV, generator=torch.Generator(DEV).manual_seed(3)).bfloat16()
    e.x[e.x == 0] = 1.0
    e.d_loss = torch.rand(slots, device=DEV)
    e.d_loss[3] = float("inf")
    dx, dt = e.loss_bwd(e.loss()[1])
    sign = torch.ones(vocab, 1, device=DEV)
    sign[e.target[3]] = -1
    assert torch.equal(dt.float(), sign * e.x[3].float().sign() * float("inf"))
    finite = torch.ones(slots, dtype=torch.bool, device=DEV)
    finite[3] = False
    assert torch.isfinite(dx[finite]).all() and not torch.isfinite(dx[3]).any()
