"""Serving a fine-tuned model from a paged cache of keys and values: what is timed and compared when a kernel changes.

A case is one pass through one of two paths (`path`):

  write    s2a_cache_write of the new tokens' k and v into the cache's pages, then s2a_cache_read of the same tokens: what the cache
           now stands for.  With `e4m3` the cache holds 8-bit floats with a power of two for every token and head, else bf16.
  attend   s2a_paged_fwd: every new token attends the cached tokens of its sequence up to itself, all of them or (`window` > 0)
           the last `window` ones and the sequence's first `sinks`.

The new tokens of `B` sequences lie one after the other in one tensor [T, heads, d]; sequence b has the rows starts[b] to starts[b + 1] - 1
and, with them, lengths[b] tokens in the cache.  Of `longest` and `new` tokens the first sequence has all; the last one has the shares
1 - len_spread and 1 - new_spread, those between in even steps.  The cache is a pool of pages [pages, Hkv, page, d] for k and v each;
table[b, i] is the page of sequence b's tokens i * page to (i + 1) * page - 1.

Attention shapes are the Llama2 ones of paper_2309_12307_b200/inputs.py and of the tests; values are N(0, 1) in bf16, as everywhere in
this repository.
"""
from __future__ import annotations

import math

import torch

own = False


def _case(path, B, longest, new, H, Hkv, d, page, e4m3=False, window=0, sinks=0, len_spread=0.0, new_spread=0.0):
    return dict(path=path, B=B, longest=longest, new=new, H=H, Hkv=Hkv, d=d, page=page, e4m3=e4m3, window=window, sinks=sinks,
                len_spread=len_spread, new_spread=new_spread)


def listed():
    cases = {
        # one token of one short sequence on a small model: what a call costs
        "decode_tiny": _case("attend", 1, 1000, 1, 4, 4, 64, 16),
        # a batch of chats of very different lengths on a 7B model, one token each: the cache is read once
        "decode_7b_8k_batch": _case("attend", 16, 8192, 1, 32, 32, 128, 64, len_spread=0.9),
        # the same on a 70B model with grouped KV heads and a cache in 8 bits
        "decode_70b_32k_e4m3": _case("attend", 8, 32768, 1, 64, 8, 128, 64, e4m3=True, len_spread=0.5),
        # a single user at the literal 100,000 tokens: few rows, one very long axis
        "decode_7b_100000_e4m3": _case("attend", 1, 100000, 1, 32, 32, 128, 128, e4m3=True),
        # streaming: the first tokens and a window of the last ones; drafts of up to four tokens are checked at once
        "decode_window_drafts": _case("attend", 32, 16001, 4, 16, 4, 64, 16, window=2048, sinks=4, len_spread=0.8, new_spread=0.75),
        # a prompt taken in pieces: the last piece of 8k on a 7B model
        "chunk_7b_8k": _case("attend", 1, 8192, 2048, 32, 32, 128, 64),
        # the last piece of 32k on a 70B model from a cache in 8 bits
        "chunk_70b_32k_e4m3": _case("attend", 1, 32768, 2048, 64, 8, 128, 64, e4m3=True),
        # a piece in the middle of a long stream on a 13B model, with a window
        "chunk_13b_window": _case("attend", 1, 32768, 4096, 40, 40, 128, 128, window=8192, sinks=64),
        # a server's step: some sequences bring a prompt, others one token; odd sizes, small pages
        "mixed_ragged_gqa": _case("attend", 6, 4001, 701, 32, 8, 64, 16, len_spread=0.9, new_spread=1.0),
        # one token of each of 64 sequences goes into the cache
        "write_step_e4m3": _case("write", 64, 8192, 1, 64, 8, 128, 64, e4m3=True, len_spread=0.9),
        # a whole prompt piece, quantised
        "write_chunk_7b_e4m3": _case("write", 2, 16384, 8192, 32, 32, 128, 128, e4m3=True, new_spread=0.3),
        # ragged prompts into a bf16 cache with small pages
        "write_ragged_bf16": _case("write", 6, 6001, 4003, 16, 4, 64, 16, len_spread=0.3, new_spread=0.7),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "drafts", "chunk", "mixed", "write"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 16, 32, 40])
    rep = rng.choice([r for r in (1, 1, 2, 3, 4, 7, 8) if r * Hkv <= 64])
    longest = _log_uniform(rng, 1, 65536)
    new = 1 if kind == "decode" else min(longest, rng.randint(2, 8) if kind == "drafts" else _log_uniform(rng, 9, 4096))
    B = 1 if kind == "chunk" else _log_uniform(rng, 1, 64)
    e4m3 = rng.random() < 0.5
    # no more than the largest listed case: bytes of the cache, pairs of rows and keys, new values
    while B > 1 and (B * longest * Hkv * d > 16 * 8192 * 32 * 128 or B * longest * new * rep * Hkv > 32768 * 2048 * 64 or B * new * Hkv * d > 1 << 26):
        B = (B + 1) // 2
    while longest * Hkv * d > 16 * 8192 * 32 * 128 or longest * new * rep * Hkv > 32768 * 2048 * 64:
        longest = (longest + 1) // 2
        new = min(new, longest)
    window = _log_uniform(rng, 1, max(2, longest)) if kind != "write" and rng.random() < 0.3 else 0
    return _case("write" if kind == "write" else "attend", B, longest, new, rep * Hkv, Hkv, d, rng.choice([16, 32, 64, 128]), e4m3=e4m3,
                 window=window, sinks=rng.choice([0, 1, 4, 64, 200]) if window else 0, len_spread=round(rng.uniform(0, 0.95), 3),
                 new_spread=1.0 if kind == "mixed" else round(rng.uniform(0, 0.9), 3) if kind in ("drafts", "write") else 0.0)


def _sizes(case):
    """New tokens and lengths of the sequences."""
    B = case["B"]
    share = [b / (B - 1) if B > 1 else 0.0 for b in range(B)]
    lengths = [max(1, case["longest"] - int(case["longest"] * case["len_spread"] * s)) for s in share]
    new = [max(1, min(n, case["new"] - int(case["new"] * case["new_spread"] * s))) for s, n in zip(share, lengths)]
    return new, lengths


def _power(e):
    """2^e in 32 bits, exactly (-126 <= e <= 127)."""
    return ((e.int() + 127) << 23).view(torch.float32)[..., None]


def _row_exponents(x):
    """The power of two of every row of d values: the least e >= -126 with max |x| <= 448 * 2^e."""
    mantissa, e = torch.frexp(x.abs().amax(-1))  # max |x| = mantissa * 2^e, 0.5 <= mantissa < 1
    return torch.where(mantissa == 0, torch.full_like(e, -126), (e - 9 + (mantissa > 0.875)).clamp(min=-126))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, Hkv, d, page = (case[k] for k in ("B", "H", "Hkv", "d", "page"))
    new, lengths = _sizes(case)
    T, width = sum(new), -(-max(lengths) // page)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)

    # the pages of a pool in use lie in no order
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    starts = torch.tensor([0] + [sum(new[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
    s = dict(case=case, table=table, starts=starts, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), T=T, most=max(new),
             reach=width * page, k_exp=None, v_exp=None)
    for x in ("k", "v"):
        pool = normal(pages, Hkv, page, d)
        if case["e4m3"]:
            e = _row_exponents(pool.float())
            pool = (pool.float() * _power(-e)).to(torch.float8_e4m3fn)
            s[x + "_exp"] = e.to(torch.int8)
        s[x + "_pool"] = pool
    if case["path"] == "write":
        s["k"], s["v"] = normal(T, Hkv, d), normal(T, Hkv, d)
    else:
        s["q"] = normal(T, H, d)
    return s


def _positions(s):
    """The sequence of each new token, and its position there."""
    rows = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["starts"][1:], rows, right=True)
    return b, s["lengths"][b].long() - s["starts"][b + 1].long() + rows


def _plain_write(s):
    case, page = s["case"], s["case"]["page"]
    b, pos = _positions(s)
    at, slot = s["table"][b, pos // page].long(), pos % page
    out = {}
    for x in ("k", "v"):
        pool = s[x + "_pool"]
        if case["e4m3"]:
            e = _row_exponents(s[x].float())
            pool.view(torch.uint8)[at, :, slot] = (s[x].float() * _power(-e)).to(torch.float8_e4m3fn).view(torch.uint8)
            s[x + "_exp"][at, :, slot] = e.to(torch.int8)
            out[x] = (pool.view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float() * _power(s[x + "_exp"][at, :, slot])).to(torch.bfloat16)
        else:
            pool[at, :, slot] = s[x]
            out[x] = pool[at, :, slot]
    return out


def _plain_attend(s):
    case = s["case"]
    B, H, Hkv, d = (case[k] for k in ("B", "H", "Hkv", "d"))
    rep, most, reach = H // Hkv, s["most"], s["reach"]

    def cached(x):
        values = s[x + "_pool"].view(torch.uint8)[s["table"].long()].view(s[x + "_pool"].dtype).float()
        if case["e4m3"]:
            values = values * _power(s[x + "_exp"][s["table"].long()])
        return values.permute(0, 2, 1, 3, 4).reshape(B, Hkv, reach, d)

    # every sequence gets `most` rows; those it has not got repeat its last one
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.minimum(torch.arange(most, device="cuda"), new[:, None] - 1)
    rows = s["starts"][:-1, None].long() + i
    pos = (s["lengths"].long() - new)[:, None] + i
    key = torch.arange(reach, device="cuda")
    seen = key <= pos[..., None]
    if case["window"]:
        seen &= (key > pos[..., None] - case["window"]) | (key < case["sinks"])
    q = s["q"].float()[rows].view(B, most, Hkv, rep, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, rep * most, d)
    score = (q @ cached("k").transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(B, Hkv, rep, most, reach)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    o = (score.view(B, Hkv, rep * most, reach) @ cached("v")).view(B, Hkv, rep, most, d) / total
    lse = (top + total.log())[..., 0]
    out = torch.empty((s["T"], H, d), dtype=torch.bfloat16, device="cuda")
    out[rows] = o.permute(0, 3, 1, 2, 4).reshape(B, most, H, d).to(torch.bfloat16)
    out_lse = torch.empty((H, s["T"]), device="cuda")
    out_lse[:, rows] = lse.permute(1, 2, 0, 3).reshape(H, B, most)
    return {"o": out, "lse": out_lse}


def run(state):
    if not own:
        return _plain_write(state) if state["case"]["path"] == "write" else _plain_attend(state)
    from paper_2309_12307_b200 import binding

    case = state["case"]
    cache = binding.PagedCache(state["k_pool"], state["v_pool"], state["k_exp"], state["v_exp"])
    where = state["table"], state["starts"], state["lengths"]
    if case["path"] == "write":
        binding.s2a_cache_write(cache, state["k"], state["v"], *where)
        k, v = binding.s2a_cache_read(cache, *where, tokens=state["T"])
        return {"k": k, "v": v}
    o, lse = binding.s2a_paged_fwd(state["q"], cache, *where, max_new=state["most"], window=case["window"], sinks=case["sinks"])
    return {"o": o, "lse": lse}


def work(case):
    new, lengths = _sizes(case)
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    T = sum(new)
    row = d + 1 if case["e4m3"] else 2 * d  # bytes of a token of a head in the cache
    if case["path"] == "write":
        # k and v are read and written into the cache, the cache is read and k and v are written
        return {"bytes": 2 * T * Hkv * (2 * 2 * d + 2 * row), "flops": 0}
    pairs = keys = 0
    for n, length in zip(new, lengths):
        first = length - n
        if case["window"]:
            low = max(0, first - case["window"] + 1)  # the first key in the window of the first new token
            keys += length - low + min(case["sinks"], low)
            for p in range(first, length):
                low = max(0, p - case["window"] + 1)
                pairs += p + 1 - low + min(case["sinks"], low)
        else:
            keys += length
            pairs += n * first + n * (n + 1) // 2
    return {"bytes": 2 * keys * Hkv * row + 2 * 2 * T * H * d + 4 * T * H, "flops": 4 * d * H * pairs}


def _scaled(x, e):
    """x * 2^e in 64 bits."""
    return x * ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, exponents):
    """What 8-bit floats stand for: sign, four bits of exponent with bias 7, three of mantissa, times 2^e."""
    x = codes.view(torch.uint8).long()
    power, fraction = (x >> 3) & 15, (x & 7).double() / 8
    size = torch.where(power == 0, fraction * 2.0 ** -6, _scaled(1 + fraction, power - 7))
    return _scaled(torch.where(x >= 128, -size, size), exponents.long()[..., None])


def _exact_rounded(x):
    """Rows of d values to 8-bit floats with a power of two: the nearest, ties to the even one."""
    x = x.double()
    e = torch.ceil(torch.log2(x.abs().amax(-1) / 448)).clamp(min=-126).long()[..., None]
    y = _scaled(x, -e)
    step = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).long() - 3
    return _scaled(torch.round(_scaled(y, -step)), step + e)


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] == "write":
        return {x: _exact_rounded(s[x]) if case["e4m3"] else s[x].double() for x in ("k", "v")}
    new, lengths = _sizes(case)
    H, Hkv, d, page = (case[k] for k in ("H", "Hkv", "d", "page"))
    o = torch.empty((s["T"], H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((H, s["T"]), dtype=torch.float64, device="cuda")
    at = 0
    for b in range(case["B"]):
        n, length = new[b], lengths[b]
        pages = s["table"][b, :-(-length // page)].long()
        query = torch.arange(length - n, length, device="cuda")[:, None]
        keys = torch.arange(length, device="cuda")[None]
        hidden = keys > query
        if case["window"]:
            hidden = hidden | ((query - keys >= case["window"]) & (keys >= case["sinks"]))
        for hk in range(Hkv):
            def of(x):
                pool = s[x + "_pool"][pages, hk]
                pool = _exact_values(pool, s[x + "_exp"][pages, hk]) if case["e4m3"] else pool.double()
                return pool.reshape(-1, d)[:length]

            k, v = of("k"), of("v")
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                score = (s["q"][at:at + n, h].double() @ k.T) / math.sqrt(d)
                score[hidden] = -math.inf
                lse[h, at:at + n] = torch.logsumexp(score, -1)
                o[at:at + n, h] = torch.exp(score - lse[h, at:at + n, None]) @ v
        at += n
    return {"o": o, "lse": lse}
