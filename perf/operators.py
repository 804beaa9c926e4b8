"""The operators at the two ends of a model on one context-parallel rank's slots, as cases that can be timed: the lookup of
the slots' rows in the vocabulary table and its gradient, and the cross entropy of the slots' next tokens over the
whole vocabulary with its gradient.

A case is a dict of plain values.  `what` says which call one pass makes:

  embed        rows of the table for the tokens of the slots
  embed_grad   gradient of the table from the gradients of the rows: the whole table, or added to one that is there
  loss         cross entropy of the slots (evaluation)
  train        cross entropy, then the gradients of rows and table (training)

`docs` tokens in documents of a length between `lo` and `hi` (their logarithms uniform) are divided among `cp` ranks, every
document into 2 * cp chunks of which a rank has two; the slots of rank `rank` are what the pass works on, padding
among them.  Token frequencies fall as 1 / rank of the word, as in text.
"""
import math

import numpy as np
import torch

own = False


def _case(name, what, docs, lo, hi, cp, rank, vocab, hidden, scale=1.0, doc_seed=1, add=False, masked=0.0):
    return dict(name=name, what=what, docs=docs, lo=lo, hi=hi, cp=cp, rank=rank, vocab=vocab, hidden=hidden, scale=scale,
                doc_seed=doc_seed, add=add, masked=masked)


def listed():
    return [
        # lookup for one of eight ranks of a 128K-token micro-batch, rows scaled by the root of their length
        _case("embed_128k_cp8", "embed", 131072, 64, 65536, 8, 3, 131072, 4096, scale=64.0, doc_seed=2),
        # the smallest call: a few dozen tokens of one short document
        _case("embed_small", "embed", 61, 61, 61, 1, 0, 32768, 1024, doc_seed=3),
        # gradient of the whole table for the same rank
        _case("embed_grad_128k_cp8", "embed_grad", 131072, 64, 65536, 8, 3, 65536, 4096, scale=64.0, doc_seed=2),
        # a table shared with the loss: gradient added to what the loss left there; an odd number of words, one rank
        _case("embed_grad_tied_8k", "embed_grad", 8191, 64, 1536, 1, 0, 50001, 1024, scale=32.0, doc_seed=7, add=True),
        # a short micro-batch of tiny documents on one of two ranks
        _case("embed_grad_small", "embed_grad", 700, 1, 64, 2, 1, 32768, 1024, doc_seed=4),
        # evaluation of one of eight ranks of a 128K-token micro-batch
        _case("loss_128k_cp8", "loss", 131072, 64, 65536, 8, 3, 65536, 4096, doc_seed=2),
        # evaluation of a 4K-token micro-batch of short documents, odd sizes
        _case("loss_4k_odd", "loss", 4095, 64, 1536, 1, 0, 50001, 1544, doc_seed=5),
        # evaluation of one short answer: latency of few rows against the whole table
        _case("loss_few_rows", "loss", 45, 45, 45, 1, 0, 65536, 2048, doc_seed=6, masked=0.5),
        # training step of one of eight ranks of a 128K-token micro-batch: the main case, and the largest
        _case("train_128k_cp8", "train", 131072, 64, 65536, 8, 3, 65536, 4096, doc_seed=2),
        # a whole micro-batch of 8K tokens on one rank, the prompts' tokens not trained on, odd number of words
        _case("train_8k_masked", "train", 8192, 64, 1536, 1, 0, 50001, 2048, doc_seed=8, masked=0.4),
        # the small-document regime: documents of 1 to 64 tokens on one of four ranks, most slots padding
        _case("train_tiny_docs_cp4", "train", 16384, 1, 64, 4, 1, 32768, 1024, scale=0.5, doc_seed=4),
        # one short document, where the table is read and written for a few rows
        _case("train_few_rows", "train", 33, 33, 33, 1, 0, 32768, 1024, doc_seed=9),
    ]


_MOST = 6.0 * 16384 * 65536 * 4096          # operations of the largest case


def draw(rng):
    while True:
        what = rng.choice(["embed", "embed_grad", "loss", "loss", "train", "train"])
        tokens = int(math.exp(rng.uniform(math.log(1), math.log(131072))))
        cp = rng.choice([1, 1, 2, 4, 8])
        lo, hi = rng.choice([(1, 64), (64, 1536), (64, 65536), (tokens, tokens)])
        vocab = int(math.exp(rng.uniform(math.log(512), math.log(140000))))
        vocab = rng.choice([vocab, vocab // 64 * 64])
        hidden = rng.choice([8, 32, 64]) * rng.randint(1, 64)
        case = _case("", what, tokens, min(lo, tokens), min(hi, tokens), cp, rng.randrange(cp), vocab, hidden, scale=rng.choice([1.0, 1.0, 0.5, 0.37, 16.0 if "embed" in what else 0.8]),
                     doc_seed=rng.randrange(1, 10**6), add=what == "embed_grad" and rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.3]))
        del case["name"]
        if _labelled(case)[2] and work(case)["flops"] <= _MOST and vocab * hidden <= 65536 * 4096:
            return case


def _maps(case):
    """Lengths' offsets and the rank's slots: global token of each, -1 where a chunk reaches beyond its document."""
    rng = np.random.default_rng(case["doc_seed"])
    lens = []
    left = case["docs"]
    while left > 0:
        n = min(left, int(round(math.exp(rng.uniform(math.log(case["lo"]), math.log(case["hi"]))))))
        lens.append(n)
        left -= n
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    cp, rank = case["cp"], case["rank"]
    if cp == 1:
        return cu, np.arange(cu[-1])
    slots = []
    for start, n in zip(cu[:-1], lens):
        c = -(-n // (2 * cp))
        for chunk in (rank, 2 * cp - 1 - rank):
            at = np.arange(chunk * c, (chunk + 1) * c)
            slots.append(np.where(at < n, start + at, -1))
    return cu, np.concatenate(slots)


def _targets(case):
    """Which tokens of the packed sequence are trained on: the others (prompts) are marked in the copy that the loss reads."""
    rng = np.random.default_rng(case["doc_seed"] + 1)
    trained = np.ones(case["docs"], dtype=bool)
    if case["masked"]:
        run = 16
        trained = np.repeat(rng.random(-(-case["docs"] // run)) >= case["masked"], run)[:case["docs"]]
    return trained


def _labelled(case):
    cu, slots = _maps(case)
    last = np.zeros(case["docs"], dtype=bool)
    last[cu[1:] - 1] = True
    g = slots[slots >= 0]
    g = g[~last[g]]
    return len(slots), int((slots >= 0).sum()), int(_targets(case)[g + 1].sum())


def work(case):
    n_q, n_real, n = _labelled(case)
    v, h = case["vocab"], case["hidden"]
    if case["what"] == "embed":
        return {"bytes": 2.0 * h * (min(n_real, v) + n_q) + 4 * n_q, "flops": 0.0}
    if case["what"] == "embed_grad":
        return {"bytes": 2.0 * h * (n_real + (2 * min(n_real, v) if case["add"] else v)) + 4 * n_q, "flops": 1.0 * n_real * h}
    rows = 2.0 * h * (n + v)
    if case["what"] == "loss":
        return {"bytes": rows + 12 * n_q, "flops": 2.0 * n * v * h}
    return {"bytes": rows + 2.0 * h * (n_q + v) + 16 * n_q, "flops": 6.0 * n * v * h}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cu, slots = _maps(case)
    t, v, h = case["docs"], case["vocab"], case["hidden"]
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    # word frequencies fall as 1 / rank; which words are the frequent ones belongs to the seed
    rank = (torch.rand(t, generator=gen, device="cuda", dtype=torch.float64) * math.log(v + 1)).exp().long().clamp_(1, v) - 1
    tokens = torch.randperm(v, generator=gen, device="cuda")[rank].int()
    s = dict(case=case, tokens=tokens, q_idx=torch.from_numpy(slots.astype(np.int32)).cuda(), cu=torch.from_numpy(cu.astype(np.int32)).cuda())
    n_q = len(slots)
    if case["what"] == "embed_grad":
        s["dx"] = (normal(n_q, h) / 64).bfloat16()
        if case["add"]:
            s["dtable"] = (normal(v, h) / 64).bfloat16()
    else:
        # rows of length about 2 before scaling, as behind a last norm of rows of length sqrt(hidden)
        s["table"] = (normal(v, h) * (2 / math.sqrt(h))).bfloat16()
    if case["what"] in ("loss", "train"):
        s["targets"] = torch.where(torch.from_numpy(_targets(case)).cuda(), tokens, -100).int()
        # rows point to their target to a degree between not at all (an untrained model) and far (a word that is certain)
        g = s["q_idx"].long()
        follow = s["table"][tokens[(g + 1).clamp_(0, t - 1)].long()].float()
        sure = torch.rand(n_q, 1, generator=gen, device="cuda") * 4
        s["x"] = (normal(n_q, h) + sure * follow).bfloat16()
        s["x"][g < 0] = float("nan")      # whatever a padding slot's row holds
    if case["what"] == "train":
        # the mean over the micro-batch's tokens
        s["d_loss"] = torch.full((n_q,), 1.0 / t, device="cuda")
    if own:
        from paper_2503_17924_amd import binding as B
        s["ends"] = B.Vocabulary(slots, cu, v, h, embed_scale=case["scale"], logit_scale=case["scale"])
    return s


def _plain(s):
    case = s["case"]
    q_idx, scale, v = s["q_idx"].long(), case["scale"], case["vocab"]
    real = q_idx >= 0
    if case["what"] in ("embed", "embed_grad"):
        word = s["tokens"].long()[q_idx.clamp(min=0)]
        if case["what"] == "embed":
            return (scale * s["table"][word].float() * real[:, None]).bfloat16()
        sums = torch.zeros(v, case["hidden"], device="cuda").index_add_(0, word[real], s["dx"][real].float())
        return ((s["dtable"].float() if case["add"] else 0) + scale * sums).bfloat16()
    # target of a slot: the next token where that lies in the same document
    t = case["docs"]
    end = s["cu"].long()[torch.searchsorted(s["cu"].long(), q_idx, right=True).clamp(max=len(s["cu"]) - 1)]
    target = s["targets"].long()[(q_idx + 1).clamp(max=t - 1)]
    has = real & (q_idx + 1 < end) & (target >= 0) & (target < v)
    x, table, target = s["x"][has].float(), s["table"].float(), target[has]
    logits = scale * (x @ table.T)
    lse_rows = torch.logsumexp(logits, 1)
    at = torch.arange(len(target), device="cuda")
    loss = torch.zeros(len(q_idx), device="cuda")
    lse = torch.full((len(q_idx),), -math.inf, device="cuda")
    loss[has], lse[has] = lse_rows - logits[at, target], lse_rows
    if case["what"] == "loss":
        return loss, lse
    d = torch.exp_(logits.sub_(lse_rows[:, None]))
    d[at, target] -= 1
    d *= scale * s["d_loss"][has][:, None]
    dx = torch.zeros(len(q_idx), case["hidden"], device="cuda")
    dx[has] = d @ table
    return loss, lse, dx.bfloat16(), (d.T @ x).bfloat16()


def run(state):
    if not own:
        return _plain(state)
    s, ends, what = state, state["ends"], state["case"]["what"]
    if what == "embed":
        return ends.embed(s["tokens"], s["table"])
    if what == "embed_grad":
        # the gradient that is there stays as it is for the next pass: a pass adds to a copy of it
        return ends.embed_backward(s["tokens"], s["dx"], s["dtable"].clone(), accumulate=True) if s["case"]["add"] else ends.embed_backward(s["tokens"], s["dx"])
    loss, lse = ends.loss(s["x"], s["table"], s["targets"])
    if what == "loss":
        return loss, lse
    dx, dtable = ends.loss_backward(s["x"], s["table"], s["targets"], lse, s["d_loss"])
    return loss, lse, dx, dtable


def exact(case, seed):
    s = prepare(case, seed)
    cu, slots = _maps(case)
    v, h, scale = case["vocab"], case["hidden"], float(case["scale"])
    n_q = len(slots)
    doc = np.searchsorted(cu, slots, side="right") - 1
    tokens = s["tokens"].cpu().numpy()
    real = np.flatnonzero(slots >= 0)
    word = torch.from_numpy(tokens[slots[real]].astype(np.int64)).cuda()
    rows = torch.from_numpy(real).cuda()
    f64 = dict(device="cuda", dtype=torch.float64)
    if case["what"] == "embed":
        out = torch.zeros(n_q, h, **f64)
        out[rows] = s["table"][word].double() * scale
        return out
    if case["what"] == "embed_grad":
        out = s["dtable"].double() if case["add"] else torch.zeros(v, h, **f64)
        return out.index_add_(0, word, s["dx"][rows].double() * scale)
    targets = s["targets"].cpu().numpy()
    kept = [i for i in real.tolist() if slots[i] + 1 < cu[doc[i] + 1] and 0 <= targets[slots[i] + 1] < v]
    rows = torch.tensor(kept, dtype=torch.int64, device="cuda")
    target = torch.from_numpy(targets[slots[kept] + 1].astype(np.int64)).cuda()
    x = s["x"][rows].double()
    top, total = torch.full((len(kept),), -math.inf, **f64), torch.zeros(len(kept), **f64)
    pieces = [(a, min(a + 8192, v)) for a in range(0, v, 8192)]
    for a, b in pieces:
        logits = x @ s["table"][a:b].double().T * scale
        if not len(kept):
            break
        new = torch.maximum(top, logits.amax(1))
        total = total * torch.exp(top - new) + torch.exp(logits - new[:, None]).sum(1)
        top = new
    log_sum = top + torch.log(total)
    own_logit = (x * s["table"][target].double()).sum(1) * scale
    loss, lse = torch.zeros(n_q, **f64), torch.full((n_q,), -math.inf, **f64)
    loss[rows], lse[rows] = log_sum - own_logit, log_sum
    if case["what"] == "loss":
        return loss, lse
    weight = s["d_loss"][rows].double() * scale
    dx_rows, dtable = torch.zeros(len(kept), h, **f64), torch.zeros(v, h, **f64)
    for a, b in pieces:
        part = s["table"][a:b].double()
        prob = torch.exp(x @ part.T * scale - log_sum[:, None]) * weight[:, None]
        dx_rows += prob @ part
        dtable[a:b] = prob.T @ x
    dx_rows -= weight[:, None] * s["table"][target].double()
    dtable.index_add_(0, target, -weight[:, None] * x)
    dx = torch.zeros(n_q, h, **f64)
    dx[rows] = dx_rows
    return loss, lse, dx, dtable
