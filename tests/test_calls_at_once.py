"""Calls of one object that are under way at the same time (threads, streams, graphs) have workspaces of their own."""
import threading

import pytest
import torch

from paper_2503_17924_amd import binding as B

H, F, N = 256, 512, 700
OPERATORS = {"linear": lambda dev: B.Linear([*range(N), -1], H, F, activation="silu", device=dev), "ffn": lambda dev: B.GatedFFN([*range(N), -1], H, F, device=dev)}


def values(name, seed, dev):
    """Inputs of a forward and backward pass."""
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: (torch.randn(s, generator=g) / 16).bfloat16().to(dev)  # noqa: E731
    if name == "linear":
        return normal(N + 1, H), (normal(F, H),), normal(N + 1, F)
    return normal(N + 1, H), (normal(2 * F, H), normal(H, F)), normal(N + 1, H)


def step(op, x, weights, dy, keep=True):
    y, kept = op.forward(x, *weights, keep=keep)
    return [t for t in (y, *op.backward(x, *weights, dy, kept=kept)) if t is not None]


@pytest.mark.parametrize("name", OPERATORS)
def test_threads_have_rooms_of_their_own(name, monkeypatch):
    """Without a GPU: what the library would be given, by two threads that are both inside the call."""
    op, x, weights, dy = OPERATORS[name]("cpu"), *values(name, 1, "cpu")
    at, both = {}, threading.Barrier(2)

    def call(what, desc, tensors, workspace=None):
        at.setdefault(what, []).append((workspace.data_ptr(), workspace.numel()))
        both.wait(timeout=30)

    monkeypatch.setattr(B, "_vocab_call", call)
    threads = [threading.Thread(target=step, args=(op, x, weights, dy)) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(at) == 2
    for (first, size), (second, size2) in at.values():
        assert first + size <= second or second + size2 <= first


@pytest.mark.gpu
@pytest.mark.parametrize("name", OPERATORS)
def test_streams_and_threads(name):
    op = OPERATORS[name]("cuda:0")
    inputs = [values(name, seed, "cuda") for seed in range(3)]
    want = [step(op, *v) for v in inputs]
    torch.cuda.synchronize()
    got = [[] for _ in inputs]

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for i in range(20):
                got[k].append(step(op, *inputs[k], keep=i % 2 == 0))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(inputs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(len(g) == 20 for g in got)
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for out in g for a, b in zip(out, w))


@pytest.mark.gpu
@pytest.mark.parametrize("name", OPERATORS)
def test_graphs_replayed_side_by_side(name):
    """Two graphs of one object's calls on two streams, with eager calls of it on a third."""
    op = OPERATORS[name]("cuda:0")
    inputs = [values(name, seed, "cuda") for seed in range(3)]
    want = [[t.clone() for t in step(op, *v)] for v in inputs]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(3)]
    for v in inputs[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step(op, *v))
    for again in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
            with torch.cuda.stream(streams[2]):
                eager = step(op, *inputs[2])
        torch.cuda.synchronize()
        for o, w in zip([*outs, eager], want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
