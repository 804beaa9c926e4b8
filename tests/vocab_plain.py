"""Lookup and vocabulary loss in 64 bits, straight from their definitions, and how far the kernels may be from them.

Roundings counted: u = 2^-8 is half a step of bf16 relative to the value, e = 2^-24 of float.  Sums of n floats are off by at most
n e times the sum of the terms' magnitudes, in any order.
"""
import math

import numpy as np
import torch

U, E = 2.0 ** -8, 2.0 ** -24
# Exponentials below the smallest normal float, 2^-126, come out as 0, and so may products below it: each is off by less than that.
TINY = 2.0 ** -126


def words(tokens, q_idx, vocab):
    """The word a slot holds, -1 if none."""
    out = np.full(len(q_idx), -1, dtype=np.int64)
    for i, g in enumerate(np.asarray(q_idx).tolist()):
        if 0 <= g < len(tokens) and 0 <= tokens[g] < vocab:
            out[i] = tokens[g]
    return out


def targets(tokens, q_idx, cu, vocab):
    """The next token of a slot in its document, -1 if there is none or it is no word."""
    nxt = np.full(len(tokens), -1, dtype=np.int64)
    for a, b in zip(cu[:-1], cu[1:]):
        nxt[a:b - 1] = tokens[a + 1:b]
    out = np.full(len(q_idx), -1, dtype=np.int64)
    for i, g in enumerate(np.asarray(q_idx).tolist()):
        if 0 <= g < len(tokens) and 0 <= nxt[g] < vocab:
            out[i] = nxt[g]
    return out


def embed_bwd(word, dx, vocab, scale, dtable=None):
    """-> (dtable, bound)"""
    real = torch.from_numpy(np.flatnonzero(word >= 0)).to(dx.device)
    at = torch.from_numpy(word[word >= 0]).to(dx.device)
    rows = dx[real].double()
    zero = torch.zeros(vocab, dx.shape[1], dtype=torch.float64, device=dx.device)
    total, size = zero.index_add(0, at, rows) * scale, zero.index_add(0, at, rows.abs()) * scale
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    if dtable is not None:
        total, size = total + dtable.double(), size + dtable.double().abs()
    # the rows' sum, the product with the scale and the sum with the old value in float, one rounding to bf16
    off = (count + 3) * E * size
    return total, off + U * (total.abs() + off)


def loss(x, table, target, scale):
    """-> (loss, lse, bounds of both); x: any rows where target < 0"""
    n = len(target)
    has = torch.from_numpy(np.flatnonzero(target >= 0)).to(x.device)
    t = torch.from_numpy(target[target >= 0]).to(x.device)
    f64 = dict(dtype=torch.float64, device=x.device)
    out = [torch.zeros(n, **f64), torch.full((n,), -math.inf, **f64), torch.zeros(n, **f64), torch.zeros(n, **f64)]
    if len(t):
        xs, es = x[has].double(), table.double()
        l = scale * (xs @ es.T)
        # of a logit: the product's sum; of its exponential: the argument's product (of up to |l| + |lse|) and the function's own 2 steps
        off = (x.shape[1] * E * scale * (xs.abs() @ es.abs().T)).amax(1)
        lse = torch.logsumexp(l, 1)
        lt = l.gather(1, t[:, None])[:, 0]
        reach = l.abs().amax(1) + lse.abs() + 1
        # sum of exponentials: table.shape[0] / 16 partial sums at most, and the roundings of maximum, logarithm and result
        bound = off + (8 * reach + 8 + table.shape[0] / 16) * E
        out[0][has], out[1][has] = lse - lt, lse
        out[2][has], out[3][has] = bound + off + 4 * E * lt.abs(), bound
    return out


def loss_bwd(x, table, target, scale, d_loss):
    """-> (dx, dtable, bounds of both).  D is rounded to bf16 once.  Up to 128 slots dX has what the rounding leaves out at the targets, and up to 32 dE has
    what it leaves out everywhere, itself rounded to bf16: u * u of the value."""
    n, h = x.shape
    f64 = dict(dtype=torch.float64, device=x.device)
    dx, dtable = torch.zeros(n, h, **f64), torch.zeros(table.shape[0], h, **f64)
    dx_off, dt_off = torch.zeros_like(dx), torch.zeros_like(dtable)
    has = torch.from_numpy(np.flatnonzero(target >= 0)).to(x.device)
    t = torch.from_numpy(target[target >= 0]).to(x.device)
    if not len(t):
        return dx, dtable, dx_off, dt_off
    xs, es, g = x[has].double(), table.double(), d_loss[has].double()
    l = scale * (xs @ es.T)
    lse = torch.logsumexp(l, 1)
    p = torch.exp(l - lse[:, None])
    off = (h * E * scale * (xs.abs() @ es.abs().T)).amax(1) + 8 * (l.abs().amax(1) + lse.abs() + 2) * E
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    d = g[:, None] * scale * (p - hot)
    # the exponential's error and the lse's, then 4 float roundings, then bf16
    d_off = (g.abs() * scale)[:, None] * (p * (2 * off)[:, None] + 4 * E * (p + hot) + 2 * TINY)
    size = d.abs() * (1 + 2 * off)[:, None]
    dx[has] = d @ es
    sums = (d_off + U * size * (1 - hot if n <= 128 else 1)) @ es.abs() + (table.shape[0] + 64) * E * (d.abs() @ es.abs())
    dx_off[has] = sums + U * (dx[has].abs() + sums)
    dtable = d.T @ xs
    sums = (d_off + (U * U if n <= 32 else U) * size).T @ xs.abs() + (len(t) + 64) * E * (d.abs().T @ xs.abs())
    dt_off = sums + U * (dtable.abs() + sums)
    return dx, dtable, dx_off, dt_off


def check(name, got, want, bound):
    got, want = got.double().to(want.device), want
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    worst = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    assert not torch.isnan(worst).any(), f"{name}: not a number"
    if worst.numel():
        k = int(worst.argmax())
        assert worst.max() <= 0, f"{name}: {got.flatten()[k]} for {want.flatten()[k]} +- {bound.flatten()[k]} at {k} of {tuple(want.shape)}"
