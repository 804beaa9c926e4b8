"""Lookup and cross entropy over the vocabulary, with their gradients, against the definitions in 64 bits (vocab_plain)."""
import numpy as np
import pytest

import vocab_plain as plain
from gpu_helpers import Guarded
from oracle import shard as osh
from paper_2503_17924_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Ends:
    """One rank's problem.  Every buffer that the library writes lies between guard bands."""

    def __init__(self, seed, docs, cp, rank, vocab, hidden, scale=1.0, mode=osh.PER_DOC_PADDED, logit=2.0, masked=0.1):
        import torch
        self.torch, self.vocab, self.hidden, self.scale = torch, vocab, hidden, scale
        rng = np.random.default_rng(seed)
        sh = osh.shard(docs, cp, rank, mode)
        self.q_idx, self.cu = sh["q_idx"].astype(np.int32), sh["cu_seqlens_k"].astype(np.int32)
        self.t, self.n_q = int(self.cu[-1]), len(self.q_idx)
        # few frequent words, many rare ones, the first and the last, and values that are none
        tok = np.minimum((vocab ** rng.random(self.t)).astype(np.int64) - 1, vocab - 1)
        tok[rng.random(self.t) < 0.1] = vocab - 1
        self.tok = tok.astype(np.int32)
        other = rng.random(self.t) < masked
        self.tok[other] = rng.choice([-1, -100, vocab, 2 ** 31 - 1, -2 ** 31], size=int(other.sum()))
        g = torch.Generator(device="cpu").manual_seed(seed)
        bf = lambda *s: torch.randn(s, generator=g).to(DEV)
        self.table = (bf(vocab, hidden) * logit / np.sqrt(hidden)).bfloat16()
        self.x, self.dx = bf(self.n_q, hidden).bfloat16(), bf(self.n_q, hidden).bfloat16()
        self.d_loss = bf(self.n_q) / max(self.n_q, 1)
        self.word, self.target = plain.words(self.tok, self.q_idx, vocab), plain.targets(self.tok, self.q_idx, self.cu, vocab)
        # what a slot without a word or target holds is never used
        junk = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device=DEV)
        self.dx[torch.from_numpy(self.word < 0).to(DEV)] = junk[0].bfloat16()
        none = torch.from_numpy(np.flatnonzero(self.target < 0)).to(DEV)
        self.x[none] = junk[none % 4].bfloat16()[:, None]
        self.d_loss[none] = junk[none % 4]
        self.tokens, self.q_dev = torch.from_numpy(self.tok).to(DEV), torch.from_numpy(self.q_idx).to(DEV)
        self.cu_dev = torch.from_numpy(self.cu).to(DEV)
        self.desc = B.vocab_desc(self.n_q, self.t, len(docs), vocab, hidden, scale)
        self.add = B.vocab_desc(self.n_q, self.t, len(docs), vocab, hidden, scale, B.VOCAB_ACCUMULATE)
        self.rooms = [self.room("workspace", max(n, 1), torch.uint8) for n in B.wlb_vocab_workspace_size(self.desc)]

    def room(self, name, shape, dtype=None):
        return Guarded(self.torch, shape if isinstance(shape, tuple) else (shape,), dtype or self.torch.bfloat16, DEV, name)

    def done(self, *rooms):
        self.torch.cuda.synchronize()
        for r in (*rooms, *self.rooms):
            r.check()

    def embed(self):
        x = self.room("x", (self.n_q, self.hidden))
        B.wlb_embed_fwd(self.desc, self.tokens, self.q_dev, self.table, x.t)
        self.done(x)
        return x.t

    def embed_bwd(self, old=None):
        dt = self.room("dtable", (self.vocab, self.hidden))
        if old is not None:
            dt.t.copy_(old)
        B.wlb_embed_bwd(self.desc if old is None else self.add, self.tokens, self.q_dev, self.dx, dt.t, self.rooms[0].t)
        self.done(dt)
        return dt.t

    def loss(self):
        lo, ls = self.room("loss", self.n_q, self.torch.float32), self.room("lse", self.n_q, self.torch.float32)
        B.wlb_loss_fwd(self.desc, self.x, self.table, self.tokens, self.q_dev, self.cu_dev, lo.t, ls.t, self.rooms[1].t)
        self.done(lo, ls)
        return lo.t, ls.t

    def loss_bwd(self, lse):
        dx, dt = self.room("dx", (self.n_q, self.hidden)), self.room("dtable", (self.vocab, self.hidden))
        B.wlb_loss_bwd(self.desc, self.x, self.table, self.tokens, self.q_dev, self.cu_dev, lse, self.d_loss, dx.t, dt.t, self.rooms[2].t)
        self.done(dx, dt)
        return dx.t, dt.t

    def check_embed(self):
        got, torch = self.embed(), self.torch
        rows = torch.from_numpy(np.maximum(self.word, 0)).to(DEV)
        want = (self.table[rows].float() * torch.tensor(self.scale, device=DEV)).bfloat16()
        want[torch.from_numpy(self.word < 0).to(DEV)] = 0
        assert torch.equal(got, want), "one rounding of the float product"

    def check_embed_bwd(self):
        old = self.torch.randn(self.vocab, self.hidden, device=DEV).bfloat16()
        absent = np.ones(self.vocab, bool)
        absent[self.word[self.word >= 0]] = False
        absent = self.torch.from_numpy(absent).to(DEV)
        for o in (None, old):
            got = self.embed_bwd(o)
            plain.check("dtable of the lookup", got, *plain.embed_bwd(self.word, self.dx, self.vocab, self.desc.scale, o))
            assert self.torch.equal(got[absent], self.torch.zeros_like(got[absent]) if o is None else o[absent])
            assert self.torch.equal(got, self.embed_bwd(o)), "reproducible bit for bit"

    def check_loss(self, backward=True):
        loss, lse = self.loss()
        want = plain.loss(self.x, self.table, self.target, self.desc.scale)
        plain.check("lse", lse, want[1], want[3])
        plain.check("loss", loss, want[0], want[2])
        if not backward:
            return
        dx, dt = self.loss_bwd(lse)
        want = plain.loss_bwd(self.x, self.table, self.target, self.desc.scale, self.d_loss)
        plain.check("dx", dx, want[0], want[2])
        plain.check("dtable", dt, want[1], want[3])
        again = self.loss_bwd(lse)
        assert self.torch.equal(dx, again[0]) and self.torch.equal(dt, again[1]), "reproducible bit for bit"


# lengths of one token, tiles' edges and beyond; words and columns at the edges of tiles, steps and copies
SMALL = [
    ([1], 1, 0, 1, 8), ([2], 1, 0, 1, 8), ([2], 1, 0, 2, 8), ([3], 1, 0, 5, 16), ([33], 1, 0, 255, 64), ([34], 1, 0, 256, 72), ([31, 1, 1], 1, 0, 257, 128),
    ([65], 1, 0, 511, 136), ([64], 2, 1, 513, 200), ([129], 1, 0, 1000, 264), ([130], 1, 0, 777, 256), ([257, 1], 1, 0, 300, 520), ([300, 41, 7, 1, 1, 90], 2, 0, 2049, 328),
    ([1] * 40, 1, 0, 300, 64), ([3] * 50, 4, 1, 300, 64), ([5, 1, 700], 8, 7, 640, 1032), ([1030], 1, 0, 64, 8), ([2100, 1, 13], 1, 0, 130, 24), ([700], 1, 0, 33000, 48),
]


@pytest.mark.parametrize("docs,cp,rank,vocab,hidden", SMALL)
def test_lookup_and_its_gradient(docs, cp, rank, vocab, hidden):
    e = Ends(1, docs, cp, rank, vocab, hidden, 0.37)
    e.check_embed()
    e.check_embed_bwd()


@pytest.mark.parametrize("docs,cp,rank,vocab,hidden", SMALL)
def test_loss_and_its_gradient(docs, cp, rank, vocab, hidden):
    Ends(2, docs, cp, rank, vocab, hidden, 0.7).check_loss()


@pytest.mark.parametrize("docs,vocab,hidden", [([4096], 3, 64), ([4097], 70000, 16), ([131072], 3, 8), ([131073], 70000, 16), ([140000, 5], 600000, 8),
                                               ([30000], 5, 520), ([20000], 300, 1040), ([9000, 1], 2000, 8)])
def test_lookup_gradient_of_many_slots(docs, vocab, hidden):
    """One group of tiles and the first slot behind it; the largest list that is sorted by search and the first that is sorted by digits, one to
    three of them; words that fill hundreds of pieces."""
    e = Ends(3, docs, 1, 0, vocab, hidden, 2.0)
    e.check_embed()
    e.check_embed_bwd()


@pytest.mark.parametrize("docs,cp,rank,vocab,hidden", [([16700], 1, 0, 33000, 64), ([2600, 400], 1, 0, 16400, 776), ([5000], 1, 0, 520, 2056),
                                                       ([4900], 1, 0, 13000, 2048), ([16, 60], 1, 0, 40000, 72), ([31], 1, 0, 20000, 1032), ([9, 4], 1, 0, 70, 2048)])
def test_loss_in_pieces_and_wide_tiles(docs, cp, rank, vocab, hidden):
    """Three pieces of the vocabulary; more tiles than compute units; a long sum along few words; tiles divided so that
    their parts take two rounds; few slots and many words."""
    Ends(4, docs, cp, rank, vocab, hidden).check_loss()


@pytest.mark.parametrize("slots", [20, 60, 120])
@pytest.mark.parametrize("vocab,hidden", [(1000, 128), (1000, 192), (1000, 256), (777, 960), (70001, 192), (70001, 320), (140000, 256)])
def test_few_slots_whose_tiles_start_at_different_steps(slots, vocab, hidden):
    """Columns of two steps, of as many as there are buffers, and more; one tile to a workgroup and several."""
    Ends(5, [slots], 1, 0, vocab, hidden).check_loss()


def test_every_slot_without_a_target():
    import torch
    e = Ends(5, [1] * 70, 1, 0, 500, 64)
    loss, lse = e.loss()
    assert torch.equal(loss, torch.zeros_like(loss)) and torch.isneginf(lse).all()
    dx, dt = e.loss_bwd(lse)
    assert not dx.any() and not dt.any()
    e = Ends(5, [64], 1, 0, 500, 64, masked=1.0)
    assert not e.embed().any() and not e.embed_bwd().any()
    assert not any(t.any() for t in e.loss_bwd(e.loss()[1]))


@pytest.mark.parametrize("logit", [1e-3, 30.0, 300.0])
def test_flat_and_certain_distributions(logit):
    """Probabilities that are all alike, and such that are 0 or 1 to the last bit."""
    Ends(6, [200], 1, 0, 700, 64, logit=logit).check_loss()


def test_weights_of_one_size_are_not_rounded():
    """A factor that all slots share (1 / tokens) does not enter the rounding of the logits' gradient: 1/3 gives three times less than 1."""
    import torch
    e = Ends(7, [150], 1, 0, 400, 64)
    _, lse = e.loss()
    e.d_loss.fill_(1.0)
    one = [t.double() for t in e.loss_bwd(lse)]
    e.d_loss.fill_(1 / 3)
    for a, b in zip(one, e.loss_bwd(lse)):
        assert ((a / 3 - b.double()).abs() <= (a / 3).abs() * (2 * plain.U + plain.U ** 2) + 1e-30).all()
    e.d_loss.fill_(0.0)
    assert not any(t.any() for t in e.loss_bwd(lse))


def test_a_gradient_that_is_no_number_stays_with_its_row():
    import torch
    e = Ends(8, [150], 1, 0, 400, 64, masked=0.0)
    _, lse = e.loss()
    e.d_loss.fill_(0.5)
    e.d_loss[3] = float("inf")
    dx, _ = e.loss_bwd(lse)
    other = torch.ones(150, dtype=torch.bool, device=DEV)
    other[3] = False
    assert torch.isfinite(dx[other]).all() and not torch.isfinite(dx[3]).any()


def test_gradients_agree_with_differences():
    """Loss along a direction, forward against backward: the change of the summed loss over a small step of x and of the table."""
    import torch
    e = Ends(9, [90, 40], 1, 0, 300, 64, masked=0.0)
    e.d_loss = torch.rand(e.n_q, device=DEV)
    _, lse = e.loss()
    dx, dt = e.loss_bwd(lse)
    want = plain.loss_bwd(e.x, e.table, e.target, 1.0, e.d_loss)
    has = torch.from_numpy(e.target >= 0).to(DEV)
    h = 1e-4
    for got, off, which in ((dx, want[2], "x"), (dt, want[3], "table")):
        step = torch.randn(got.shape, dtype=torch.float64, device=DEV)
        if which == "x":
            step[~has] = 0
        ends = []
        for sign in (1, -1):
            x = e.x.double() + sign * h * step if which == "x" else e.x.double()
            table = e.table.double() + sign * h * step if which == "table" else e.table.double()
            ends.append((plain.loss(x, table, e.target, 1.0)[0] * e.d_loss.double())[has].sum())
        slope = float((ends[0] - ends[1]) / (2 * h))
        # the gradient's own error along the direction, and the differences' third-order term
        assert abs(float((got.double() * step)[has if which == "x" else slice(None)].sum()) - slope) <= float((off * step.abs()).sum()) + 1e-4 * abs(slope) + 1e-4


def test_all_ranks_together_are_the_whole_sequence():
    """A training step's run on every rank: lookup, loss, its gradient, and the lookup's gradient added to the table's; the
    ranks' losses and table gradients sum to those of the sequence on one rank."""
    import torch
    docs, vocab, hidden = [517, 3, 40, 700, 64, 1, 211], 1000, 128
    results = {}
    for cp in (1, 4):
        loss_sum, table_sum, size = 0.0, 0, 0
        for rank in range(cp):
            e = Ends(10, docs, cp, rank, vocab, hidden)
            ends = B.Vocabulary(e.q_idx, e.cu, vocab, hidden, embed_scale=8.0)
            x = ends.embed(e.tokens, e.table)
            loss, lse = ends.loss(x, e.table, e.tokens)
            d_loss = torch.full_like(loss, 1.0 / sum(docs))
            dx, dt = ends.loss_backward(x, e.table, e.tokens, lse, d_loss)
            want = plain.loss_bwd(x, e.table, e.target, 1.0, d_loss)
            plain.check("dx", dx, want[0], want[2])
            back, off = plain.embed_bwd(e.word, dx, vocab, 8.0, dt)
            assert ends.embed_backward(e.tokens, dx, dt, accumulate=True) is dt
            plain.check("dtable of both", dt, back, off)
            loss_sum += float(loss.double().sum())
            table_sum = table_sum + dt.double()
            size = size + dt.double().abs() + want[3] * 8 + want[2].sum(0) * 8
        results[cp] = loss_sum, table_sum, size
    (l1, t1, s1), (l4, t4, s4) = results[1], results[4]
    assert abs(l1 - l4) <= 1e-5 * abs(l1)
    # every rank's partial sum is rounded once per call: two roundings of up to 4 partial sums, and bf16 D and dx on either side
    assert ((t1 - t4).norm() / t1.norm()) <= 4 * 2 * plain.U


def test_captured_into_a_graph_and_replayed():
    """A step in a graph, replayed with new inputs between eager steps of the same object, equals the eager step every time."""
    import torch
    e = Ends(11, [900, 17, 300], 2, 1, 3000, 192)
    ends = B.Vocabulary(e.q_idx, e.cu, e.vocab, e.hidden, embed_scale=3.0)

    def step(out):
        x = ends.embed(e.tokens, e.table, out[0])
        ends.loss(x, e.table, e.tokens, out[1], out[2])
        ends.loss_backward(x, e.table, e.tokens, out[2], e.d_loss, out[3], out[4])
        ends.embed_backward(e.tokens, out[3], out[4], accumulate=True)

    def rooms():
        f32, bf = torch.float32, torch.bfloat16
        return [torch.empty(e.n_q, e.hidden, dtype=bf, device=DEV), torch.empty(e.n_q, dtype=f32, device=DEV), torch.empty(e.n_q, dtype=f32, device=DEV),
                torch.empty(e.n_q, e.hidden, dtype=bf, device=DEV), torch.empty(e.vocab, e.hidden, dtype=bf, device=DEV)]

    eager, kept = rooms(), rooms()
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kept)
    for k in range(4):
        e.table.copy_((torch.randn(e.vocab, e.hidden, device=DEV) / 10).bfloat16())
        e.tokens.copy_(e.tokens[torch.randperm(e.t, device=DEV)])
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for a, b in zip(kept, eager):
            bits = torch.int32 if a.dtype == torch.float32 else torch.int16        # slots whose d_loss is no number have targets now
            assert torch.equal(a.view(bits), b.view(bits)), f"replay {k}"


def test_memory_of_other_shapes_is_refused():
    import torch
    e = Ends(13, [40], 1, 0, 100, 64)
    ends = B.Vocabulary(e.q_idx, e.cu, e.vocab, e.hidden)
    loss, lse = ends.loss(e.x, e.table, e.tokens)
    for call, error in ((lambda: ends.embed(e.tokens, e.table[:50]), ValueError), (lambda: ends.embed(e.tokens.long(), e.table), TypeError),
                        (lambda: ends.embed(e.tokens, e.table.t()), TypeError), (lambda: ends.embed(e.tokens.cpu(), e.table), TypeError),
                        (lambda: ends.loss(e.x[:-1], e.table, e.tokens), ValueError), (lambda: ends.loss(e.x.float(), e.table, e.tokens), TypeError),
                        (lambda: ends.loss_backward(e.x, e.table, e.tokens, lse.double(), e.d_loss), TypeError),
                        (lambda: ends.loss_backward(e.x, e.table, e.tokens, lse, e.d_loss[None]), ValueError),
                        (lambda: ends.embed_backward(e.tokens, e.dx, accumulate=True), ValueError),
                        (lambda: ends.embed(e.tokens, torch.empty(e.vocab * e.hidden + 1, dtype=torch.bfloat16, device=DEV)[1:].view(e.vocab, e.hidden)), B.WlbError),
                        (lambda: B.wlb_loss_fwd(e.desc, e.x, e.table, e.tokens, e.q_dev, e.cu_dev, loss, lse, e.rooms[1].t[:-1]), B.WlbError)):
        with pytest.raises(error):
            call()
    with pytest.raises(B.WlbError):
        B.Vocabulary(e.q_idx, e.cu, 100, 60).embed(e.tokens, torch.empty(100, 60, dtype=torch.bfloat16, device=DEV))


def test_on_another_stream():
    import torch
    e = Ends(12, [600], 1, 0, 2000, 128)
    want = e.loss_bwd(e.loss()[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ends = B.Vocabulary(e.q_idx, e.cu, e.vocab, e.hidden)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss, lse = ends.loss(e.x, e.table, e.tokens)
        got = ends.loss_backward(e.x, e.table, e.tokens, lse, e.d_loss)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_workspace_is_kept_from_reuse_while_another_stream_works():
    import torch
    e = Ends(12, [600], 1, 0, 2000, 128)
    side = torch.cuda.Stream()
    ends = B.Vocabulary(e.q_idx, e.cu, e.vocab, e.hidden)
    ends.loss(e.x, e.table, e.tokens)                       # the workspace belongs to the current stream
    torch.cuda.synchronize()
    nbytes, at = ends.workspace[1].numel(), ends.workspace[1].data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                      # about 0.1 s
        loss, _ = ends.loss(e.x, e.table, e.tokens)
    del ends
    rooms = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(4)]
    busy = not side.query()
    side.synchronize()
    assert busy and at not in [r.data_ptr() for r in rooms]
    assert torch.equal(loss, e.loss()[0])
