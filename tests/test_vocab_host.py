"""Lookup and vocabulary loss without a GPU: argument checks, workspace sizes, and the plain forms against each other."""
import ctypes

import numpy as np
import pytest
import torch

import vocab_plain as plain
from paper_2503_17924_amd import binding as B


def refused(desc, status, call=None):
    with pytest.raises(B.WlbError) as e:
        (call or B.wlb_vocab_workspace_size)(desc)
    assert e.value.status == status and str(e.value)


@pytest.mark.parametrize("change,status", [
    (dict(n_q=0), 1), (dict(t_kv=0), 1), (dict(n_docs=0), 1), (dict(vocab=0), 1), (dict(hidden=0), 1), (dict(hidden=-8), 1),
    (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(flags=2), 1), (dict(flags=-1), 1),
    (dict(hidden=12), 3), (dict(hidden=65544), 3), (dict(vocab=2 ** 30 + 1), 3), (dict(n_q=2 ** 30 + 1), 3)])
def test_descriptors_refused(change, status):
    good = dict(n_q=5, t_kv=9, n_docs=2, vocab=100, hidden=64, scale=1.0, flags=0)
    B.wlb_vocab_workspace_size(B.vocab_desc(**good))
    refused(B.vocab_desc(**{**good, **change}), status)


def call(name, desc, pointers, workspace=0x100000, nbytes=1 << 40):
    """A C call with pointers that are never followed: every refusal comes before anything is launched."""
    args = [ctypes.c_void_p(p) for p in pointers]
    if name != "wlb_embed_fwd":
        args += [ctypes.c_void_p(workspace), ctypes.c_size_t(nbytes)]
    st = getattr(B.lib(), name)(ctypes.byref(desc), *args, None)
    return st, B.lib().wlb_last_error().decode()


# pointers of each call, the first bit of alignment that each needs
CALLS = {"wlb_embed_fwd": (4, 4, 16, 16), "wlb_embed_bwd": (4, 4, 16, 16), "wlb_loss_fwd": (16, 16, 4, 4, 4, 4, 4),
         "wlb_loss_bwd": (16, 16, 4, 4, 4, 4, 4, 16, 16)}


@pytest.mark.parametrize("name", CALLS)
def test_pointers_and_workspaces_refused(name):
    desc = B.vocab_desc(5, 9, 2, 100, 64)
    good = [0x200000 + 4096 * i for i in range(len(CALLS[name]))]
    for i, align in enumerate(CALLS[name]):
        st, text = call(name, desc, good[:i] + [0] + good[i + 1:])
        assert st == 1 and "null" in text and name in text
        st, text = call(name, desc, good[:i] + [good[i] + align // 2] + good[i + 1:])
        assert st == 1 and "misaligned" in text
    st, text = call(name, B.vocab_desc(5, 9, 2, 100, 64, 1.0, 2), good)
    assert st == 1 and "flags" in text
    if name != "wlb_embed_bwd":
        assert call(name, B.vocab_desc(5, 9, 2, 100, 64, 1.0, B.VOCAB_ACCUMULATE), good)[0] == 1
    if name == "wlb_embed_fwd":
        return
    assert call(name, desc, good, workspace=0)[0] == 1
    assert call(name, desc, good, workspace=0x100010)[0] == 1
    need = B.wlb_vocab_workspace_size(desc)[["wlb_embed_bwd", "wlb_loss_fwd", "wlb_loss_bwd"].index(name)]
    st, text = call(name, desc, good, nbytes=need - 1)
    assert st == 2 and str(need) in text


@pytest.mark.parametrize("name", ["wlb_loss_fwd", "wlb_loss_bwd"])
def test_loss_sizes_refused(name):
    good = [0x200000 + 4096 * i for i in range(len(CALLS[name]))]
    for desc in (B.vocab_desc(2 ** 20, 2 ** 20, 1, 1000, 2048), B.vocab_desc(2 ** 24, 2 ** 24, 1, 2 ** 24, 8)):
        assert call(name, desc, good)[0] == 3


def test_null_descriptor():
    for name in CALLS:
        args = [None] * (len(CALLS[name]) + (0 if name == "wlb_embed_fwd" else 1))
        args += [] if name == "wlb_embed_fwd" else [ctypes.c_size_t(0)]
        assert getattr(B.lib(), name)(None, *args, None) == 1
    assert B.lib().wlb_vocab_workspace_size(None, None, None, None) == 1


def test_workspace_does_not_grow_with_the_logits():
    """16384 slots x 131072 words: the logits in 32 bits take 8 GiB; the forward keeps 8 bytes for every 256 of them (64 MiB) and up to 128 MiB of
    partial sums, and the backward one piece."""
    e, f, b = B.wlb_vocab_workspace_size(B.vocab_desc(16384, 131072, 16, 131072, 4096))
    assert f < 2 ** 33 // 40 and b < 2 ** 31 and e < 2 ** 25


def test_tensors_of_the_host_are_refused():
    d = B.vocab_desc(2, 2, 1, 4, 8)
    i, t = torch.zeros(2, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        B.wlb_embed_fwd(d, i, i, t, t[:2])


def test_plain_targets_by_hand():
    cu, tok = [0, 3, 4, 7], np.array([5, 6, 7, 8, 9, -1, 2])
    q = [0, 1, 2, 3, 4, 5, 6, -1, 7, 100]
    assert plain.targets(tok, q, cu, 9).tolist() == [6, 7, -1, -1, -1, 2, -1, -1, -1, -1]
    assert plain.words(tok, q, 9).tolist() == [5, 6, 7, 8, -1, -1, 2, -1, -1, -1]


def test_plain_gradients_agree_with_differences():
    g = torch.Generator().manual_seed(3)
    x, table = torch.randn(5, 8, generator=g, dtype=torch.float64), torch.randn(11, 8, generator=g, dtype=torch.float64)
    target, d_loss = np.array([3, -1, 0, 10, 3]), torch.rand(5, generator=g, dtype=torch.float64)
    dx, dt, _, _ = plain.loss_bwd(x, table, target, 0.7, d_loss)
    total = lambda: float((plain.loss(x, table, target, 0.7)[0] * d_loss).sum())  # noqa: E731
    for t, grad in ((x, dx), (table, dt)):
        for k in range(t.numel()):
            at, h = np.unravel_index(k, t.shape), 1e-6
            old = float(t[at])
            t[at] = old + h
            up = total()
            t[at] = old - h
            down = total()
            t[at] = old
            assert abs((up - down) / (2 * h) - float(grad[at])) < 1e-7
