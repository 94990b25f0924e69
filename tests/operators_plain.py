"""Plain implementations, in 64 bits, of the operators around a gated, sparse block: what the tests compare the kernels with."""
import math

import torch

D = torch.float64


def norm(a, kind, eps):
    """(normalised rows, mean, 1 / sqrt(mean square + eps))"""
    mean = a.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(a[:, :1])
    rstd = 1 / torch.sqrt((a - mean).square().mean(1, keepdim=True) + eps)
    return (a - mean) * rstd, mean, rstd


def gates_of(gate, rows, per):
    return gate[torch.arange(rows, device=gate.device) // per]


def gated_norm(x, y=None, post=None, gate=None, pre=None, kind="layer", per=None, resid_scale=1.0, eps=1e-5):
    """(h, n) of 64-bit inputs; n is None without pre."""
    affine = lambda a, p: a * p[0] + (0 if p[1] is None else p[1])
    h = x
    if y is not None:
        z = y if post is None else affine(norm(y, kind, eps)[0], post)
        h = resid_scale * x + (z if gate is None else gates_of(gate, x.shape[0], per or max(x.shape[0], 1)) * z)
    return h, None if pre is None else affine(norm(h, kind, eps)[0], pre)


def dispatch(expert, experts, capacity):
    """(slot [tokens, k], ranges [experts, 2]) as lists, choice by choice."""
    tokens, k = expert.shape
    ids = expert.reshape(-1).tolist()
    lists = [[i for i, e in enumerate(ids) if e == x] for x in range(experts)] if len(ids) * experts < 200000 else None
    if lists is None:
        lists = [[] for _ in range(experts)]
        for i, e in enumerate(ids):
            if 0 <= e < experts:
                lists[e].append(i)
    slot, ranges, at = [-1] * len(ids), [], 0
    for e, mine in enumerate(lists):
        if capacity:
            mine, at = mine[:capacity], e * capacity
        for r, i in enumerate(mine):
            slot[i] = at + r
        ranges.append([at, len(mine)])
        at += len(mine)
    return torch.tensor(slot, dtype=torch.int32).reshape(tokens, k), torch.tensor(ranges, dtype=torch.int32).reshape(experts, 2)


def combine(rows, slot, weights=None, add=None):
    T, k = slot.shape
    ok = (slot >= 0) & (slot < rows.shape[0])
    w = torch.ones_like(slot, dtype=D) if weights is None else weights.to(D)
    out = torch.zeros(T, rows.shape[1], dtype=D, device=rows.device) if add is None else add.to(D).clone()
    for j in range(k):
        t = ok[:, j].nonzero().reshape(-1)
        out[t] += w[t, j, None] * rows.to(D)[slot[t, j].long()]
    return out


def adamw(master, m, v, g, lr, b1, b2, eps, t, decay=0.0, factor=1.0):
    """(master, m, v) after a step, 64 bits."""
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    step = m / (1 - b1 ** t) / (torch.sqrt(v / (1 - b2 ** t)) + eps)
    return master - lr * factor * (step + decay * master), m, v


def e4m3_half_step(x):
    """Half the distance between the e4m3 neighbours of x, 64 bits: 2^-4 of its power of two, 2^-10 below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    return 2.0 ** (e - 4)


def half_step(dtype):
    """The relative error of one rounding to the nearest."""
    return torch.finfo(dtype).eps / 2


U32 = 2.0 ** -24
assert math.isclose(half_step(torch.float32), U32)
