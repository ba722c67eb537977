"""Norms of queries and keys for each head and the rotation of positions, from their definitions, in 64 bits on the CPU (test infrastructure only).

A row is the d values of one head of a token.  `radians` are the frequencies of the rotated pairs; the first 2 * len(radians) values of a row are rotated.
"""
from __future__ import annotations

import torch


def pairs(d: int, n: int, interleaved: bool):
    """Places of the first and of the second values of the n pairs."""
    i = torch.arange(n)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + n)


def turned(x, positions, radians, interleaved, backwards=False):
    """x [T, heads, d]: pair i of token t as a complex number, times e^(i positions[t] radians[i])."""
    x = x.double().clone()
    u, v = pairs(x.shape[-1], len(radians), interleaved)
    angle = positions.double()[:, None] * torch.as_tensor(radians, dtype=torch.float64)
    c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if backwards else 1)
    a, b = x[..., u], x[..., v]
    x[..., u], x[..., v] = a * c - b * s, a * s + b * c
    return x


def rotate(x, positions, radians, interleaved=False, weight=None, eps=None):
    x = x.double()
    if eps is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            x = x * weight.double()
    return turned(x, positions, radians, interleaved)


def rotate_bwd(x, dy, positions, radians, interleaved=False, weight=None, eps=None):
    """Gradients of x and of the norm's weight (None without a norm), of sum(rotate(x) * dy)."""
    g = turned(dy, positions, radians, interleaved, backwards=True)
    if eps is None:
        return g, None
    x = x.double()
    size = (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x / size
    wg = g if weight is None else g * weight.double()
    return (wg - n * (wg * n).mean(-1, keepdim=True)) / size, (g * n).sum((0, 1))


def reach(x, dims: int, n: int, interleaved: bool):
    """Of every value, the sum of the magnitudes of its pair: what errors of an angle are relative to."""
    size = x.double().abs().clone()
    u, v = pairs(dims, n, interleaved)
    both = size[..., u] + size[..., v]
    size[..., u], size[..., v] = both, both
    return size
