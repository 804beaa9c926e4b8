"""Gradients of the loss where few of the slots have a target: what decides is how many have one, not how many slots there are."""
import numpy as np
import pytest

import vocab_plain as plain
from paper_2503_17924_amd import binding as B
from test_vocab_gpu import DEV, Ends

pytestmark = pytest.mark.gpu


def keep(e, slots):
    """Leaves the tokens behind `slots` in the sequence and makes the others none; rows and weights without a target hold what they like."""
    import torch
    tok = np.full_like(e.tok, -1)
    at = e.q_idx[slots] + 1
    tok[at] = e.tok[at]
    e.tok, e.target = tok, plain.targets(tok, e.q_idx, e.cu, e.vocab)
    e.tokens = torch.from_numpy(tok).to(DEV)
    none = torch.from_numpy(e.target < 0).to(DEV)
    e.x[none], e.d_loss[none] = float("nan"), float("inf")
    return e


def check(e):
    """Against the bounds of a call that has the labelled slots alone."""
    import torch
    has = np.flatnonzero(e.target >= 0)
    rows = torch.from_numpy(has).to(DEV)
    x, target, weight = e.x[rows], e.target[has], e.d_loss[rows]
    loss, lse = e.loss()
    want = plain.loss(x, e.table, target, e.desc.scale)
    plain.check("lse", lse[rows], want[1], want[3])
    plain.check("loss", loss[rows], want[0], want[2])
    dx, dt = e.loss_bwd(lse)
    want = plain.loss_bwd(x, e.table, target, e.desc.scale, weight)
    plain.check("dtable", dt, want[1], want[3])
    # rows of dx have nothing to do with each other: their bound is that of a call of few slots, however many there are
    for k in range(0, len(has), 128):
        few = plain.loss_bwd(x[k:k + 128], e.table, target[k:k + 128], e.desc.scale, weight[k:k + 128])
        plain.check("dx", dx[rows[k:k + 128]], few[0], few[2])
    none = torch.from_numpy(e.target < 0).to(DEV)
    assert not loss[none].any() and torch.isneginf(lse[none]).all() and not dx[none].any()
    again = e.loss_bwd(lse)
    assert torch.equal(dx, again[0]) and torch.equal(dt, again[1]), "reproducible bit for bit"


# slots; then words and columns for which D, dtable and dx have tiles of each kind, whole and divided
@pytest.mark.parametrize("labelled", [1, 3, 32, 33])
@pytest.mark.parametrize("docs,vocab,hidden", [([45], 300, 64), ([70], 3000, 192), ([128], 777, 1032), ([200], 700, 264), ([200], 1000, 4104), ([300, 1, 900], 5000, 1032),
                                               ([1500], 70000, 200), ([2500], 900, 3000)])
def test_few_labelled_slots_among_many(docs, vocab, hidden, labelled):
    rng = np.random.default_rng(labelled)
    e = Ends(21, docs, 1, 0, vocab, hidden, 0.9, masked=0.0)
    has = np.flatnonzero(e.target >= 0)
    check(keep(e, rng.permutation(has)[:labelled]))


@pytest.mark.parametrize("cp,rank", [(2, 1), (4, 0)])
def test_few_labelled_slots_among_padding(cp, rank):
    e = Ends(22, [1, 2, 3, 1, 40, 1, 1, 5, 2, 600], cp, rank, 2000, 136, masked=0.0)
    check(keep(e, np.flatnonzero(e.target >= 0)[:7]))


def test_a_short_answer_behind_a_long_prompt_in_pieces():
    """Three pieces of the vocabulary, targets in each of them."""
    e = Ends(23, [16700], 1, 0, 33000, 64, masked=0.0)
    want = [np.flatnonzero((e.target >= a) & (e.target < b))[-2:] for a, b in ((0, 15000), (17000, 32000), (32800, 33000))]
    assert all(len(w) == 2 for w in want)
    check(keep(e, np.concatenate(want)))


@pytest.mark.parametrize("slots", [50, 129, 700])
@pytest.mark.parametrize("vocab,hidden", [(40, 264), (2000, 264), (700, 8)])
def test_rows_whose_gradient_is_their_target_alone(slots, vocab, hidden):
    """Every row of the table but the target's is 0, so the rounding of D at the target would be the whole of dx's error, on top of its own: up to 128 or not."""
    import torch
    e = Ends(24, [slots + 1], 1, 0, vocab, hidden, masked=0.0)
    e.tok[:] = 0
    e.target[:-1] = 0
    e.tokens.fill_(0)
    e.table[1:] = 0
    row = e.table[0].double()
    sure = torch.linspace(-1, 2, slots + 1, device=DEV, dtype=torch.float64)[:, None] * np.log(vocab)
    noise = torch.randn(slots + 1, hidden, device=DEV, dtype=torch.float64, generator=torch.Generator(DEV).manual_seed(1)) / 50
    e.x = (sure * row / (row @ row) + noise).bfloat16()
    e.d_loss.fill_(1.0)
    check(e)


def test_graph_whose_replays_have_few_many_and_no_targets():
    """What a captured call launches does not depend on how many slots have a target."""
    import torch
    e = Ends(26, [700], 1, 0, 3000, 136, masked=0.0)
    full, weight = e.tok.copy(), torch.rand(e.n_q, device=DEV)
    e.x.nan_to_num_(1.0)
    e.d_loss.copy_(weight)
    ends = B.Vocabulary(e.q_idx, e.cu, e.vocab, e.hidden, logit_scale=0.8)
    f32, bf = torch.float32, torch.bfloat16
    loss, lse = torch.empty(e.n_q, dtype=f32, device=DEV), torch.empty(e.n_q, dtype=f32, device=DEV)
    dx, dt = torch.empty(e.n_q, e.hidden, dtype=bf, device=DEV), torch.empty(e.vocab, e.hidden, dtype=bf, device=DEV)

    def step():
        ends.loss(e.x, e.table, e.tokens, loss, lse)
        ends.loss_backward(e.x, e.table, e.tokens, lse, e.d_loss, dx, dt)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for labelled in (5, 699, 0, 32, 33, 128, 1):
        tok = np.full_like(full, -1)
        at = np.random.default_rng(labelled).permutation(699)[:labelled] + 1
        tok[at] = full[at]
        e.tokens.copy_(torch.from_numpy(tok))
        for t in (loss, lse, dx, dt):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        target = plain.targets(tok, e.q_idx, e.cu, e.vocab)
        has = np.flatnonzero(target >= 0)
        rows = torch.from_numpy(has).to(DEV)
        want = plain.loss_bwd(e.x[rows], e.table, target[has], 0.8, weight[rows])
        plain.check(f"dx, {labelled}", dx[rows], want[0], want[2])
        plain.check(f"dtable, {labelled}", dt, want[1], want[3])
        replayed = [t.clone() for t in (loss, lse, dx, dt)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (loss, lse, dx, dt))), labelled
