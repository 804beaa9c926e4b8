"""Sizes at which the vocabulary calls change what they launch: another sort, more rows than one launch has threads for."""
import numpy as np
import pytest

from paper_2503_17924_amd import binding as B
from test_vocab_gpu import DEV, Ends

pytestmark = pytest.mark.gpu
GIB = 1 << 30


def room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * GIB:
        pytest.skip(f"{gib} GiB of device memory")


@pytest.mark.parametrize("docs,vocab,hidden", [([53248], 70000, 8), ([53249], 70000, 8), ([53249], 3, 64), ([40000, 30000], 300000, 72), ([100000], 32767, 16)])
def test_lookup_gradient_around_the_largest_list_that_is_sorted_by_search(docs, vocab, hidden):
    Ends(61, docs, 1, 0, vocab, hidden, 2.0).check_embed_bwd()


def test_lookup_of_more_slots_than_a_launch_has_threads_for():
    """A row takes 128 threads, four rows at a time: 2^27 slots are 2^32 threads."""
    import torch
    room(160)
    n_q, t_kv, vocab, hidden = 2 ** 27 + 5, 1000, 300, 520
    g = torch.Generator(DEV).manual_seed(1)
    table = torch.randn(vocab, hidden, device=DEV, generator=g).bfloat16()
    tokens = torch.randint(-1, vocab, (t_kv,), device=DEV, generator=g, dtype=torch.int32)
    q_idx = torch.randint(-1, t_kv, (n_q,), device=DEV, generator=g, dtype=torch.int32)
    x = torch.empty(n_q, hidden, dtype=torch.bfloat16, device=DEV)
    for a in range(0, n_q, 2 ** 23):
        x[a:a + 2 ** 23].view(torch.int16).fill_(-1)
    B.wlb_embed_fwd(B.vocab_desc(n_q, t_kv, 1, vocab, hidden), tokens, q_idx, table, x)
    for a in range(0, n_q, 2 ** 21):
        q = q_idx[a:a + 2 ** 21].long()
        word = torch.where(q >= 0, tokens[q.clamp(min=0)].long(), -1)
        assert torch.equal(x[a:a + 2 ** 21], table[word.clamp(min=0)] * (word >= 0)[:, None]), a
    del x
    torch.cuda.empty_cache()


def test_lookup_gradient_of_the_largest_table():
    """2^30 words, all but a few of them absent: every row is written."""
    import torch
    room(24)
    vocab, hidden = 2 ** 30, 8
    words = [0, 1, 63, 64, 2 ** 26 - 1, 2 ** 26, 2 ** 29 + 7, vocab - 2, vocab - 1, vocab - 1]
    n = len(words)
    tokens, q_idx = torch.tensor(words, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    desc = B.vocab_desc(n, n, 1, vocab, hidden)
    dx = torch.randn(n, hidden, device=DEV).bfloat16()
    dtable = torch.empty(vocab, hidden, dtype=torch.bfloat16, device=DEV)
    for a in range(0, vocab, 2 ** 26):
        dtable[a:a + 2 ** 26].view(torch.int16).fill_(-1)
    B.wlb_embed_bwd(desc, tokens, q_idx, dx, dtable, torch.empty(B.wlb_vocab_workspace_size(desc)[0], dtype=torch.uint8, device=DEV))
    at = torch.tensor(words[:-1], device=DEV)
    want = torch.cat([dx[:-2], (dx[-2].float() + dx[-1].float()).bfloat16()[None]])
    assert torch.equal(dtable[at], want)
    dtable[at] = 0
    for a in range(0, vocab, 2 ** 26):
        assert not dtable[a:a + 2 ** 26].view(torch.int16).any(), a
    del dtable
    torch.cuda.empty_cache()


def test_loss_of_more_slots_than_a_launch_has_threads_for():
    """2^26 slots, a wavefront to each; a few have a target, among them the last but one."""
    import torch
    room(48)
    n_q, vocab, hidden = 2 ** 26 + 3, 200, 8
    has = np.array([0, 70, 2 ** 22 - 1, 2 ** 22, 2 ** 25 + 11, n_q - 2])
    tokens = torch.full((n_q,), -1, dtype=torch.int32, device=DEV)
    target = torch.arange(len(has), device=DEV) * 37 % vocab
    at = torch.from_numpy(has).to(DEV)
    tokens[at + 1] = target.int()
    q_idx, cu = torch.arange(n_q, dtype=torch.int32, device=DEV), torch.tensor([0, n_q], dtype=torch.int32, device=DEV)
    x = torch.full((n_q, hidden), float("nan"), dtype=torch.bfloat16, device=DEV)
    x[at] = torch.randn(len(has), hidden, device=DEV).bfloat16()
    table = torch.randn(vocab, hidden, device=DEV).bfloat16()
    desc = B.vocab_desc(n_q, n_q, 1, vocab, hidden)
    workspace = torch.empty(max(B.wlb_vocab_workspace_size(desc)[1:]), dtype=torch.uint8, device=DEV)
    loss, lse = torch.empty(n_q, device=DEV), torch.empty(n_q, device=DEV)
    B.wlb_loss_fwd(desc, x, table, tokens, q_idx, cu, loss, lse, workspace)
    dx, dtable = torch.full_like(x, float("nan")), torch.empty_like(table)
    B.wlb_loss_bwd(desc, x, table, tokens, q_idx, cu, lse, torch.ones_like(loss), dx, dtable, workspace)
    xs, es = x[at].double().requires_grad_(), table.double().requires_grad_()
    want = torch.nn.functional.cross_entropy(xs @ es.T, target, reduction="none")
    want.sum().backward()
    assert torch.allclose(loss[at].double(), want, rtol=1e-5, atol=1e-5)
    # D's roundings, up to 2^-8 of each of its entries, whose magnitudes sum to less than 2 a row, and the output's own
    size = 2 * 2.0 ** -8 * float(table.double().abs().max()) + 2.0 ** -8 * xs.grad.abs() + 1e-5
    assert ((dx[at].double() - xs.grad).abs() <= size).all()
    assert ((dtable.double() - es.grad).abs() <= 2.0 ** -8 * es.grad.abs() + 2.0 ** -15 * float(xs.detach().abs().max()) * len(has) + 1e-5).all()
    loss[at], dx[at] = 0, 0
    assert not loss.any() and not dx.any()
    del x, dx, workspace
    torch.cuda.empty_cache()


@pytest.mark.parametrize("slots", [20, 200])
@pytest.mark.parametrize("hidden", [32776, 33024, 65528, 65536])
def test_widest_rows(slots, hidden):
    """As many tiles of columns as half of the compute units, one more, and as many as all."""
    e = Ends(62, [slots], 1, 0, 300, hidden, masked=0.0)
    e.check_embed()
    e.check_embed_bwd()
    e.check_loss()


def test_loss_of_the_largest_vocabulary():
    """2^30 words, four pieces; one slot with a target.  The definition in 64 bits, a part of the words at a time."""
    import torch
    room(60)
    vocab, hidden, part = 2 ** 30, 8, 2 ** 24
    g = torch.Generator(DEV).manual_seed(7)
    table = torch.empty(vocab, hidden, dtype=torch.bfloat16, device=DEV)
    for a in range(0, vocab, part):
        table[a:a + part] = torch.randn(part, hidden, device=DEV, generator=g).bfloat16()
    x = torch.randn(2, hidden, device=DEV, generator=g).bfloat16()
    target = vocab - 3
    tokens = torch.tensor([5, target], dtype=torch.int32, device=DEV)
    q_idx, cu = torch.arange(2, dtype=torch.int32, device=DEV), torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    desc = B.vocab_desc(2, 2, 1, vocab, hidden)
    workspace = torch.empty(max(B.wlb_vocab_workspace_size(desc)[1:]), dtype=torch.uint8, device=DEV)
    loss, lse = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    B.wlb_loss_fwd(desc, x, table, tokens, q_idx, cu, loss, lse, workspace)
    weight = torch.tensor([0.75, float("nan")], device=DEV)
    dx, dtable = torch.full_like(x, float("nan")), torch.empty_like(table)
    B.wlb_loss_bwd(desc, x, table, tokens, q_idx, cu, lse, weight, dx, dtable, workspace)
    row = x[0].double()
    sums = torch.stack([torch.exp((table[a:a + part].double() * row).sum(1)).sum() for a in range(0, vocab, part)])
    true = torch.log(sums.sum())
    own = float(table[target].double() @ row)
    # a logit is off by its eight products, a part's sum by up to 128 terms in a row and the lse by the parts that a thread adds up, 2^16
    off = (2 ** 16 + 256) * 2.0 ** -24
    assert abs(float(lse[0]) - float(true)) <= off and abs(float(loss[0]) - (float(true) - own)) <= off + 1e-5
    assert float(loss[1]) == 0 and float(lse[1]) == -float("inf") and not dx[1].any()
    want_dx, size = torch.zeros(hidden, dtype=torch.float64, device=DEV), torch.zeros(hidden, dtype=torch.float64, device=DEV)
    for a in range(0, vocab, part):
        e = table[a:a + part].double()
        d = 0.75 * torch.exp((e * row).sum(1) - true)
        size += (d[:, None] * e.abs()).sum(0)
        if a <= target < a + part:
            d[target - a] -= 0.75
        want_dx += (d[:, None] * e).sum(0)
        want = d[:, None] * row
        # D and what bf16 leaves out of it: 2^-16; the probability's error and the lse's; the output's rounding
        assert ((dtable[a:a + part].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -15 + 2 * off)).all(), a
    # D in bf16 but for the target; sums of up to 2^16 products of 32 words in a row
    assert ((dx[0].double() - want_dx).abs() <= 2.0 ** -8 * want_dx.abs() + (2.0 ** -8 + 3 * off) * size).all()
    del table, dtable, workspace
    torch.cuda.empty_cache()
