"""Formulas of the router, the moves to experts and back and the cross entropy in 64
bits, for the tests of layer_experts.py, with elementwise bounds where rounding matters
(layer_reference has the units and the blocks of the experts)."""
import math

import torch

from layer_reference import TINY, U


def route(logits, k, normalise, scale):
    """(index, weight) of the k largest logits in falling order, of equal ones the first."""
    l = logits.double().cpu()
    index = torch.full((l.shape[0], k), -1, dtype=torch.int32)
    weight = torch.zeros(l.shape[0], k, dtype=torch.float64)
    for t, row in enumerate(l.tolist()):
        # NaN above everything, both zeros alike
        order = sorted((e for e in range(len(row)) if row[e] != -math.inf),
                       key=lambda e: (0 if row[e] != row[e] else 1, 0.0 if row[e] != row[e] else -row[e], e))[:k]
        if not order:
            continue
        p = torch.softmax(l[t], 0)
        w = torch.softmax(l[t, order], 0) if normalise else p[order]
        index[t, :len(order)] = torch.tensor(order, dtype=torch.int32)
        weight[t, :len(order)] = scale * w
    return index, weight


def route_weight(logits, index, normalise, scale):
    """The weights as a function of the logits, for given choices (differentiable)."""
    there = (index >= 0) & (index < logits.shape[1])
    at = torch.where(there, index, 0).long()
    live = logits > -math.inf
    own = torch.where(there, logits.gather(1, at), -math.inf) if normalise else logits
    top = own.detach().amax(1, keepdim=True).clamp_min(-1e300)
    e = torch.where(live, torch.exp(torch.where(live, logits - top, 0.0).clamp_max(0.0)), 0.0)
    taken = torch.where(there, e.gather(1, at), 0.0)
    total = taken.sum(1, keepdim=True) if normalise else e.sum(1, keepdim=True)
    return scale * torch.where(there, taken / torch.where(total > 0, total, 1.0), 0.0)


def route_back(dweight, logits, index, normalise, scale):
    """dlogits by the formula, and the magnitudes that it adds up."""
    l, dw = logits.double(), scale * dweight.double()
    there = (index >= 0) & (index < l.shape[1])
    at = torch.where(there, index, 0).long()
    q = route_weight(l, index, normalise, 1.0)
    dw = torch.where(there, dw, 0.0)
    mean, size = (q * dw).sum(1, keepdim=True), (q * dw.abs()).sum(1, keepdim=True)
    if normalise:
        own, much = q * (dw - mean), q * (dw.abs() + size)
        base = big = torch.zeros_like(l)
    else:
        own, much = q * dw, q * dw.abs()
        p = torch.where(l > -math.inf, torch.softmax(l, 1), 0.0).nan_to_num(0.0)
        base, big = -p * mean, p * size
    zero = lambda v: torch.where(there, v, 0.0)
    return base.scatter_add(1, at, zero(own)), big.scatter_add(1, at, zero(much))


def sort_by_expert(index, experts):
    """(offsets, row) choice by choice."""
    flat = index.reshape(-1).tolist()
    lists = [[] for _ in range(experts)]
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            lists[e].append(i)
    offsets, row = [0], [-1] * len(flat)
    for choices in lists:
        for n, i in enumerate(choices):
            row[i] = offsets[-1] + n
        offsets.append(offsets[-1] + len(choices))
    return torch.tensor(offsets, dtype=torch.int32), torch.tensor(row, dtype=torch.int32).view(index.shape)


def combine(ys, row, weight):
    """(y, the magnitudes added up)."""
    row = row.reshape(-1, row.shape[-1]).long()
    there = (row >= 0) & (row < ys.shape[0])
    each = torch.where(there[..., None], ys.double()[torch.where(there, row, 0)], 0.0)
    if weight is not None:
        each = each * torch.where(there, weight.double().reshape(row.shape), 0.0)[..., None]
    return each.sum(1), each.abs().sum(1)


def cross_entropy(x, w, target, ignore, typ, dloss=None, grad_typ=None):
    """{name: (value, bound)} of loss, lse, dx and dw.

    A logit's sum of K products in 32 bits is off by at most K 2^-23 of the magnitudes.
    An exponential exp(-z) is off by (z + 4) 2^-24 of itself, at most 2^-17 for the z up to 100
    that matter; each is added in a chain of fewer than 100 additions and scaled by fewer than 100
    exponentials of sums that together are no larger, so the sum is off by less than
    2^-15 of itself."""
    x, w, target = x.double(), w.double(), target.long()
    counted = target != ignore
    at = torch.where(counted, target, 0)[:, None]
    D, T = x.shape[1], x.shape[0]
    l, bl = x @ w.T, D * 2.0 ** -23 * (x.abs() @ w.abs().T)
    lse = torch.logsumexp(l, 1)
    most = bl.amax(1)
    blse = most + 2.0 ** -15 + 2.0 ** -22 * lse.abs()
    picked = l.gather(1, at)[:, 0]
    loss = torch.where(counted, lse - picked, 0.0)
    bloss = torch.where(counted, blse + bl.gather(1, at)[:, 0] + 2.0 ** -23 * (lse.abs() + picked.abs()), 0.0)
    out = {"lse": (lse, blse), "loss": (loss, bloss)}
    if dloss is None:
        return out
    x = torch.where(counted[:, None], x, 0.0)
    dl = torch.where(counted, dloss.double().expand(T), 0.0)[:, None]
    p = torch.exp(l - lse[:, None])
    g = p.scatter_add(1, at, torch.full_like(dl, -1.0)) * dl
    # float16 rounds g after a power of two that brings the largest dloss to 2^10 and more
    least = TINY[typ] * (float(dl.abs().max()) * 2.0 ** -10 if typ is torch.float16 else 1.0)
    off = (bl + blse[:, None] + 2.0 ** -15)
    bg = dl.abs() * (p * off * torch.exp(off) + 2.0 ** -23) + U[typ] * g.abs() + least
    bg = torch.where(counted[:, None], bg, 0.0)
    for name, v, b, t in (("dx", g @ w, (bg + w.shape[0] * 2.0 ** -23 * g.abs()) @ w.abs(), typ),
                          ("dw", g.T @ x, (bg + T * 2.0 ** -23 * g.abs()).T @ x.abs(), grad_typ or typ)):
        out[name] = v, b * (1 + U[t]) + U[t] * v.abs() + TINY[t]
    return out
