"""Forward against backward by differences of the kernel's own losses, and the ranks' results against those of the whole sequence, entry by entry."""
import numpy as np
import pytest

import vocab_plain as plain
from paper_2503_17924_amd import binding as B
from test_vocab_gpu import DEV, Ends

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("docs,vocab,hidden", [([30], 300, 64), ([90, 40], 1000, 136), ([600, 1], 300, 64)])
@pytest.mark.parametrize("which", ["x", "table"])
def test_differences_of_the_loss(which, docs, vocab, hidden):
    """x or the table moved by a step to either side.  All operands are multiples of 2^-6 below 2, which bf16 holds, so the step is exact."""
    import torch
    e = Ends(51, docs, 1, 0, vocab, hidden, masked=0.0)
    grid = lambda t, s: (t.double() * s).mul(16).round().div(16).clamp(-1.5, 1.5)  # noqa: E731
    has = torch.from_numpy(e.target >= 0).to(DEV)
    g = torch.Generator(DEV).manual_seed(5)
    x, table = grid(torch.randn(e.n_q, hidden, device=DEV, generator=g), 1), grid(torch.randn(vocab, hidden, device=DEV, generator=g), 4 / hidden ** 0.5)
    e.d_loss = torch.rand(e.n_q, device=DEV, generator=g) + 0.5
    weight = e.d_loss.double() * has
    step = (torch.randint(0, 2, (x if which == "x" else table).shape, device=DEV, generator=g) * 2 - 1).double() / 64
    sides, exact, off = [], [], 0
    for sign in (1, -1):
        xs, ts = (x + sign * step, table) if which == "x" else (x, table + sign * step)
        e.x, e.table = xs.bfloat16(), ts.bfloat16()
        assert torch.equal(e.x.double(), xs) and torch.equal(e.table.double(), ts)
        want = plain.loss(xs, ts, e.target, 1.0)
        sides.append((e.loss()[0].double() * weight).sum())
        exact.append((want[0] * weight).sum())
        off = off + (want[2] * weight).sum()
    e.x, e.table = x.bfloat16(), table.bfloat16()
    dx, dt = e.loss_bwd(e.loss()[1])
    want = plain.loss_bwd(x, table, e.target, 1.0, e.d_loss)
    got, true, bound = (dx, want[0], want[2]) if which == "x" else (dt, want[1], want[3])
    # what a difference leaves out of a slope (its third-order term), from the definition; then the losses' and the gradient's own errors
    curved = exact[0] - exact[1] - 2 * (true * step).sum()
    tolerance = curved.abs() + off + 2 * (bound * step.abs()).sum()
    slope = 2 * (got.double() * step).sum()
    assert (sides[0] - sides[1] - slope).abs() <= tolerance
    size = 2 * (true.abs() * step.abs()).sum()
    assert tolerance <= size / 20, "the tolerance would hide a wrong gradient"


def test_ranks_sum_to_the_whole_sequence_entry_by_entry():
    import torch
    docs, vocab, hidden = [517, 3, 40, 700, 64, 1, 211], 1000, 128
    whole = None
    for cp in (1, 2, 4):
        zero = lambda: torch.zeros(vocab, hidden, dtype=torch.float64, device=DEV)  # noqa: E731
        total, exact, bound, loss_sum, loss_exact, loss_off = zero(), zero(), zero(), 0.0, 0.0, 0.0
        for rank in range(cp):
            e = Ends(52, docs, cp, rank, vocab, hidden)
            ends = B.Vocabulary(e.q_idx, e.cu, vocab, hidden, embed_scale=8.0)
            x = ends.embed(e.tokens, e.table)
            loss, lse = ends.loss(x, e.table, e.tokens)
            d_loss = torch.full_like(loss, 1.0 / sum(docs))
            dx, dt = ends.loss_backward(x, e.table, e.tokens, lse, d_loss)
            _, off = plain.embed_bwd(e.word, dx, vocab, 8.0, dt)
            ends.embed_backward(e.tokens, dx, dt, accumulate=True)
            total += dt.double()
            want = plain.loss_bwd(x, e.table, e.target, 1.0, d_loss)
            real = torch.from_numpy(np.flatnonzero(e.word >= 0)).to(DEV)
            word = torch.from_numpy(e.word[e.word >= 0]).to(DEV)
            exact += want[1].index_add(0, word, 8 * want[0][real])
            # of the two roundings of the sum; of the loss's gradients that went into it
            bound += off + want[3].index_add(0, word, 8 * want[2][real])
            of_loss = plain.loss(x, e.table, e.target, 1.0)
            loss_sum, loss_exact = loss_sum + float(loss.double().sum()), loss_exact + float(of_loss[0].sum())
            loss_off += float(of_loss[2].sum())
        assert abs(loss_sum - loss_exact) <= loss_off
        plain.check(f"dtable of {cp} ranks", total, exact, bound)
        if whole is None:
            whole = exact, loss_exact
        assert torch.allclose(exact, whole[0], rtol=1e-9, atol=1e-12) and abs(loss_exact - whole[1]) <= 1e-9 * whole[1]
