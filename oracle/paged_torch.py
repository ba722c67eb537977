"""The paged cache and its attention from their definitions, in 64 bits on the CPU (test infrastructure only).

A cache is a dict of pools: k, v [pages, Hkv, page_size, d] as floats of any type, or as uint8 codes with exponents k_exp, v_exp
[pages, Hkv, page_size].  Sequence b has rows starts[b] to starts[b+1] - 1, the last of its lengths[b] cached tokens.
"""
from __future__ import annotations

import math

import torch

NOT_FINITE = -128


def code_values():
    """The values of the 256 codes of an 8-bit float with 4 bits of exponent (bias 7) and 3 of fraction."""
    out = []
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        x = math.ldexp(f / 8, -6) if e == 0 else math.ldexp(1 + f / 8, e - 7)
        out.append(math.nan if c & 127 == 127 else -x if c >= 128 else x)
    return torch.tensor(out, dtype=torch.float64)


def row_exponent(row) -> int:
    """The least e >= -126 with max |x| <= 448 * 2^e; NOT_FINITE for a row with an infinity or a NaN."""
    row = row.double()
    if not torch.isfinite(row).all():
        return NOT_FINITE
    most, e = float(row.abs().max()), -126
    while most > math.ldexp(448.0, e):
        e += 1
    return e


def quantised_row(row):
    """(codes, e) of one row: every value to the nearest code times 2^e, of two equally near ones to the one that ends on an even bit.
    Codes that would stand for 2^128 are not taken."""
    e = row_exponent(row)
    if e == NOT_FINITE:
        return None, e
    values = code_values()[:127]
    if e == 120:
        values = values[values <= 240]
    x = row.double().abs() * math.ldexp(1.0, -e)
    x = x.clamp(max=float(values[-1]))
    above = torch.searchsorted(values, x).clamp(max=len(values) - 1)
    below = (above - 1).clamp(min=0)
    up, down = values[above] - x, x - values[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    code = torch.where(values[above] == x, above, code)
    return torch.where(torch.signbit(row.double()), code + 128, code).to(torch.uint8), e


def cached(cache, x, page, hk, slot):
    """What the cache holds for one token of one KV head."""
    row = cache[x][page, hk, slot]
    if row.dtype != torch.uint8:
        return row.double()
    e = int(cache[x + "_exp"][page, hk, slot])
    return torch.full(row.shape, math.nan, dtype=torch.float64) if e == NOT_FINITE else code_values()[row.long()] * math.ldexp(1.0, e)


def sequence_values(cache, x, table, b, length):
    """[Hkv, length, d] of sequence b."""
    page = cache[x].shape[2]
    pages = table[b, :-(-length // page)].long()
    rows = cache[x][pages]
    if rows.dtype == torch.uint8:
        e = cache[x + "_exp"][pages].double()
        values = code_values()[rows.long()] * torch.exp2(torch.where(e == NOT_FINITE, torch.full_like(e, math.nan), e))[..., None]
    else:
        values = rows.double()
    return values.transpose(0, 1).reshape(cache[x].shape[1], -1, cache[x].shape[3])[:, :length]


def visible(position, length, window, sinks):
    """The cached tokens that the token at `position` attends, as a mask over `length` of them."""
    j = torch.arange(length)
    seen = j <= position
    if window:
        seen &= (j > position - window) | (j < sinks)
    return seen


def paged_fwd(q, cache, table, starts, lengths, scale, window=0, sinks=0):
    """o, lse and, for error bounds, the sum of weight * |v| and (0 unless the cache has exponents) the largest product, over the blocks of 128
    keys, of the largest weight and the largest power of two of v in the block.  Rows of no sequence are NaN."""
    T, H, d = q.shape
    o = torch.full((T, H, d), math.nan, dtype=torch.float64)
    size, lse = o.clone(), torch.full((H, T), math.nan, dtype=torch.float64)
    largest = torch.zeros((T, H), dtype=torch.float64)
    for b in range(len(lengths)):
        row0, n, length = int(starts[b]), int(starts[b + 1] - starts[b]), int(lengths[b])
        if n == 0:
            continue
        k, v = (sequence_values(cache, x, table, b, length) for x in ("k", "v"))
        rep = H // k.shape[0]
        blocks = -(-length // 128)
        powers = None
        if "v_exp" in cache:
            page = cache["v"].shape[2]
            e = cache["v_exp"][table[b, :-(-length // page)].long()].double().transpose(0, 1).reshape(k.shape[0], -1)[:, :length]
            powers = torch.full((k.shape[0], blocks * 128), -1e9, dtype=torch.float64)
            powers[:, :length] = e
            powers = torch.exp2(powers.view(k.shape[0], blocks, 128).amax(-1))
        for i in range(n):
            seen = visible(length - n + i, length, window, sinks)
            for h in range(H):
                s = scale * (k[h // rep][seen] @ q[row0 + i, h].double())
                lse[h, row0 + i] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[h, row0 + i])
                o[row0 + i, h] = w @ v[h // rep][seen]
                size[row0 + i, h] = w @ v[h // rep][seen].abs()
                if powers is not None:
                    of_block = torch.zeros(blocks * 128, dtype=torch.float64)
                    of_block[:length][seen] = w
                    largest[row0 + i, h] = (of_block.view(blocks, 128).amax(-1) * powers[h // rep]).max()
    return o, lse, size, largest
