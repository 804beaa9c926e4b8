"""Loss and gradients where the vocabulary is taken in pieces: whole and divided tiles that add to what earlier pieces left."""
import numpy as np
import pytest

import vocab_plain as plain
from test_vocab_gpu import DEV, Ends

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,hidden", [(16400, 1032), (16400, 4104), (33100, 1024)])
def test_wide_tiles_over_pieces(vocab, hidden):
    """Two or three pieces (the last of 16 words, and of 332); 330 tiles of dX and more, most of them whole; a depth along hidden that is divided."""
    Ends(41, [16700], 1, 0, vocab, hidden).check_loss()


@pytest.mark.parametrize("slots", [128, 65, 300])
def test_few_slots_over_pieces(slots):
    """Targets in the first, a middle and the last piece: what bf16 leaves out at a target is kept until the last."""
    import torch
    vocab = {128: 2 ** 21 + 100, 65: 2 ** 22 + 60, 300: 2 ** 20 + 1000}[slots]
    e = Ends(42, [slots], 1, 0, vocab, 8, masked=0.0)
    tok = np.random.default_rng(3).integers(0, vocab, size=slots)
    tok[::3] = vocab - 1 - np.arange(len(tok[::3])) % 50
    tok[1::3] = np.arange(len(tok[1::3])) % 7
    e.tok, e.tokens = tok.astype(np.int32), torch.from_numpy(tok).int().to(DEV)
    e.target = plain.targets(e.tok, e.q_idx, e.cu, vocab)
    e.d_loss = torch.rand(slots, device=DEV)
    loss, lse = e.loss()
    want = plain.loss(e.x, e.table, e.target, 1.0)
    plain.check("lse", lse, want[1], want[3])
    plain.check("loss", loss, want[0], want[2])
    dx, dt = e.loss_bwd(lse)
    del want
    want = plain.loss_bwd(e.x, e.table, e.target, 1.0, e.d_loss)
    plain.check("dx", dx, want[0], want[2])
    plain.check("dtable", dt, want[1], want[3])
    again = e.loss_bwd(lse)
    assert torch.equal(dx, again[0]) and torch.equal(dt, again[1]), "reproducible bit for bit"
    del want
    torch.cuda.empty_cache()
