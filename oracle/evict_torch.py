"""Weights of cached tokens and eviction by them, from their definitions, in 64 bits on the CPU (test infrastructure only).  Caches are those of paged_torch.py."""
from __future__ import annotations

import math

import torch

from .paged_torch import sequence_values


def attends(positions, length: int, window: int, sinks: int):
    """[rows, length]: whether a token at each of the positions attends each key."""
    p, j = positions[:, None], torch.arange(length)[None]
    return (j <= p) & ((j > p - window) | (j < sinks) if window else torch.ones_like(j <= p))


def paged_weights(q, lse, cache, table, starts, lengths, received, before, scale, window=0, sinks=0):
    """(received, written): what it is after the call, in 64 bits, and which of its entries the call writes."""
    out, written = received.double().clone(), torch.zeros(received.shape, dtype=torch.bool)
    Hkv, page = cache["k"].shape[1], cache["k"].shape[2]
    rep = q.shape[1] // Hkv
    for b in range(len(lengths)):
        row0, end, length = int(starts[b]), int(starts[b + 1]), int(lengths[b])
        n = end - row0
        if n == 0:
            continue
        k = sequence_values(cache, "k", table, b, length)
        mask = attends(torch.arange(length - n, length), length, window, sinks)
        places = mask.any(0).nonzero()[:, 0]
        pages = table[b].long()[places // page]
        for hk in range(Hkv):
            total = torch.zeros(length, dtype=torch.float64)
            for h in range(hk * rep, (hk + 1) * rep):
                s = scale * (q[row0:end, h].double() @ k[hk].T)
                total += torch.where(mask, torch.exp(s - lse[h, row0:end, None].double()), 0.0).sum(0)
            if before is not None:
                old = places < length - n
                total[places[old]] += before[pages[old], hk, places[old] % page].double()
            out[pages, hk, places % page] = total[places]
            written[pages, hk, places % page] = True
    return out, written


def kept_tokens(weights, budget: int, sinks: int, recent: int):
    """Places of the tokens of one head that stay, ascending; `weights` of its n tokens."""
    n = len(weights)
    if n <= budget:
        return list(range(n))
    always = set(range(sinks)) | set(range(n - recent, n))
    between = [j for j in range(n) if j not in always]
    between.sort(key=lambda j: (-math.inf, j) if math.isnan(weights[j]) else (-weights[j], j))
    first_nan = [j for j in between if math.isnan(weights[j])]
    others = [j for j in between if not math.isnan(weights[j])]
    return sorted(always | set((first_nan + others)[:budget - len(always)]))


def evict(received, table, lengths, page: int, budget: int, sinks: int, recent: int):
    """kept [B][Hkv] lists of places."""
    out = []
    for b, n in enumerate(int(x) for x in lengths):
        places = torch.arange(n)
        pages = table[b].long()[places // page]
        out.append([kept_tokens(received[pages, hk, places % page].tolist(), budget, sinks, recent) for hk in range(received.shape[1])])
    return out
