"""Around the paged cache: rotating queries and keys to their positions, weighing cached tokens, and evicting them.

A case is one pass through one of five paths (`path`):

  rotate      s2a_rotate: q [T, H, d] and k [T, Hkv, d], each head's row normalised where `norm` is set (1 / root mean square, times a
              learned weight), its first `r` values rotated by the token's position.  Positions are interpolated by `scale`.
  rotate_bwd  s2a_rotate_bwd: the gradients of q and k, and with `norm` of the two weights.
  enter       s2a_rotate_write: the same for new tokens of B sequences that are served; q comes back rotated, k goes into the cache's
              pages rotated and v as it is.  s2a_cache_read then brings back what the cache stands for.
  weigh       s2a_paged_weights: the attention weight that every cached token gets from the new ones, all query heads of its KV head
              together, added to what it had before (`add`) or by itself.
  evict       s2a_cache_evict: of every sequence and KV head `budget` tokens are kept, the first `sinks`, the last `recent` and the heaviest
              others, and go to other pages in their order.  Of an 8-bit cache s2a_cache_read then brings back what was kept.

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

BASE, EPS = 10000.0, 1e-5


def _rotation(path, T, H, Hkv, d, norm=False, r=None, pairs=False, packed=False, scale=1.0, first=0):
    return dict(path=path, T=T, H=H, Hkv=Hkv, d=d, norm=norm, r=d if r is None else r, pairs=pairs, packed=packed, scale=scale, first=first)


def _cached(path, B, longest, new, H, Hkv, d, page, e4m3=False, len_spread=0.0, new_spread=0.0, **more):
    return dict(path=path, B=B, longest=longest, new=new, H=H, Hkv=Hkv, d=d, page=page, e4m3=e4m3, len_spread=len_spread, new_spread=new_spread, **more)


def listed():
    cases = {
        # a layer's queries and keys in fine-tuning a 7B model at 32k, positions interpolated to the 4096 it was trained on
        "rotate_7b_32k": _rotation("rotate", 32768, 32, 32, 128, scale=0.125),
        # a small model with norms on a ragged prompt, out of the projection's packed output
        "rotate_norm_packed": _rotation("rotate", 4001, 16, 4, 64, norm=True, packed=True),
        # the gradients of a 70B model's layer with norms
        "rotate_bwd_70b_norm": _rotation("rotate_bwd", 8192, 64, 8, 128, norm=True, scale=0.5),
        # half of each head rotated, neighbours as pairs, no norm, few tokens
        "rotate_bwd_half_pairs": _rotation("rotate_bwd", 701, 16, 16, 64, r=32, pairs=True),
        # one token for each of 16 sequences far beyond what the cache keeps: what a call costs
        "enter_step_7b": _cached("enter", 16, 2048, 1, 32, 32, 128, 64, len_spread=0.5, norm=False, scale=0.25, ahead=98000),
        # a piece of a prompt of a 70B model into 8 bits, with norms
        "enter_chunk_70b_e4m3": _cached("enter", 2, 8192, 4001, 64, 8, 128, 64, e4m3=True, new_spread=0.3, norm=True, scale=1.0, ahead=0),
        # one token for each of a batch of chats of very different lengths on a 7B model
        "weigh_step_7b": _cached("weigh", 16, 8192, 1, 32, 32, 128, 64, len_spread=0.9, window=0, sinks=0, add=True),
        # the same on a 70B model with grouped KV heads and a cache in 8 bits
        "weigh_step_70b_e4m3": _cached("weigh", 8, 32768, 1, 64, 8, 128, 64, e4m3=True, len_spread=0.5, window=0, sinks=0, add=True),
        # the last piece of a prompt of 8k on a 7B model: what it attends decides what stays
        "weigh_chunk_7b": _cached("weigh", 1, 8192, 2048, 32, 32, 128, 64, window=0, sinks=0, add=False),
        # a server's step: some sequences bring a prompt, others one token; odd sizes, small pages, a window
        "weigh_mixed_window": _cached("weigh", 6, 4001, 701, 32, 8, 64, 16, len_spread=0.9, new_spread=1.0, window=2048, sinks=4, add=True),
        # a batch of chats cut down to a quarter
        "evict_7b_batch": _cached("evict", 16, 8192, 0, 32, 32, 128, 64, len_spread=0.7, budget=2048, sinks=4, recent=512),
        # a single user's 100,000 tokens of a 70B model, from 8 bits to 8 bits
        "evict_70b_100000_e4m3": _cached("evict", 1, 100000, 0, 64, 8, 128, 64, e4m3=True, budget=8191, sinks=64, recent=1000),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    path = rng.choice(["rotate", "rotate_bwd", "enter", "weigh", "weigh", "weigh", "evict", "evict"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8, 16, 32, 40])
    H = Hkv * rng.choice([r for r in (1, 1, 2, 3, 4, 7, 8) if r * Hkv <= 64])
    scale = rng.choice([1.0, 0.5, 0.25, 0.125])
    if path in ("rotate", "rotate_bwd"):
        T = min(_log_uniform(rng, 1, 65536), 32768 * 64 * 128 // ((H + Hkv) * d))
        return _rotation(path, T, H, Hkv, d, norm=rng.random() < 0.5, r=rng.choice([d, d, d // 2, d // 4]), pairs=rng.random() < 0.3,
                         packed=rng.random() < 0.3, scale=scale, first=rng.choice([0, 0, _log_uniform(rng, 1, 100000)]))
    page, e4m3 = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    B, longest, len_spread = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 65536), round(rng.uniform(0, 0.95), 3)
    new = 0
    if path == "enter":
        new = rng.choice([1, _log_uniform(rng, 1, 4096)])
    elif path == "weigh":
        new = rng.choice([1, 1, rng.randint(2, 8), _log_uniform(rng, 9, 2048)])
        if new > 8 and rng.random() < 0.5:
            B = 1
    # no more than the largest listed cases: values of the cache, of the new tokens, pairs of rows and keys
    while B > 1 and (B * longest * Hkv * d > 16 * 8192 * 32 * 128 or B * longest * new * H > 8192 * 2048 * 32 or B * new * H * d > 1 << 25):
        B = (B + 1) // 2
    while longest * Hkv * d > 16 * 8192 * 32 * 128 or longest * min(new, longest) * H > 8192 * 2048 * 32:
        longest = (longest + 1) // 2
    new = min(new, longest)
    shape = (B, longest, new, H, Hkv, d, page)
    if path == "enter":
        return _cached(path, *shape, e4m3=e4m3, len_spread=len_spread, new_spread=round(rng.uniform(0, 0.9), 3), norm=rng.random() < 0.5, scale=scale,
                       ahead=rng.choice([0, _log_uniform(rng, 1, 100000)]))
    if path == "weigh":
        window = _log_uniform(rng, 1, max(2, longest)) if rng.random() < 0.3 else 0
        return _cached(path, *shape, e4m3=e4m3, len_spread=len_spread, new_spread=rng.choice([0.0, 1.0, round(rng.uniform(0, 0.9), 3)]) if new > 1 else 0.0,
                       window=window, sinks=rng.choice([0, 1, 4, 64, 200]) if window else 0, add=rng.random() < 0.5)
    budget = _log_uniform(rng, 1, max(1, longest // 2))
    sinks = min(rng.choice([0, 1, 4, 64]), budget)
    return _cached(path, *shape, e4m3=e4m3, len_spread=len_spread, budget=budget, sinks=sinks, recent=min(rng.choice([0, 1, 32, budget // 4]), budget - sinks))


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


def _frequencies(r, scale):
    """Radians that pair i turns by from one position to the next, in 64 bits."""
    return scale * BASE ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)


def _turns(frequencies):
    """The same in units of 2^-64 of a full turn."""
    turns = frequencies / (2 * math.pi)
    high = torch.floor(torch.ldexp(turns, torch.tensor(32, device="cuda")))
    low = torch.round(torch.ldexp(torch.ldexp(turns, torch.tensor(32, device="cuda")) - high, torch.tensor(32, device="cuda")))
    return (high.long() << 32) + low.long()


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _norm_weights(g, s, d):
    """Learned weights of the norms, about one."""
    for x in ("q", "k"):
        s[x + "_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)


def _prepare_rotation(case, g):
    T, H, Hkv, d = (case[k] for k in ("T", "H", "Hkv", "d"))
    frequencies = _frequencies(case["r"], case["scale"])
    s = dict(case=case, frequencies=frequencies, turns=_turns(frequencies), q_weight=None, k_weight=None,
             positions=torch.arange(case["first"], case["first"] + T, dtype=torch.int32, device="cuda"))
    if case["packed"]:
        qkv = _normal(g, T, H + 2 * Hkv, d)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + Hkv]
    else:
        s["q"], s["k"] = _normal(g, T, H, d), _normal(g, T, Hkv, d)
    if case["norm"]:
        _norm_weights(g, s, d)
    if case["path"] == "rotate_bwd":
        s["dq_out"], s["dk_out"] = _normal(g, T, H, d), _normal(g, T, Hkv, d)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["path"] in ("rotate", "rotate_bwd"):
        return _prepare_rotation(case, g)
    B, H, Hkv, d, page = (case[k] for k in ("B", "H", "Hkv", "d", "page"))
    new, lengths = _sizes(case)
    if case["path"] == "evict":
        new = [min(n, case["budget"]) for n in lengths]  # what the cache holds afterwards: its rows are read back
    T, width = sum(new), -(-max(lengths) // page)
    need = [-(-n // page) for n in lengths]
    kept = [-(-n // page) if case["path"] == "evict" else 0 for n in new]
    pages = sum(need) + sum(kept) + 3

    # the pages of a pool in use lie in no order; a table's unused entries name a page that nothing uses
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    spare = int(order[-1])
    table = torch.full((B, width), spare, dtype=torch.int32, device="cuda")
    to_table = torch.full((B, max(1, max(kept))), spare, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        to_table[b, :kept[b]] = order[at + need[b]:at + need[b] + kept[b]]
        at += need[b] + kept[b]
    starts = torch.tensor([0] + [sum(new[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
    s = dict(case=case, table=table, starts=starts, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), T=T, most=max(new),
             reach=width * page, spare=spare, k_exp=None, v_exp=None, q_weight=None, k_weight=None)
    for x in ("k", "v"):
        pool = _normal(g, pages, Hkv, page, d)
        if case["e4m3"]:
            e = _row_exponents(pool.float())
            pool = (pool.float() * _power(-e)).to(torch.float8_e4m3fn)
            s[x + "_exp"] = e.to(torch.int8)
        s[x + "_pool"] = pool
    if case["path"] == "enter":
        s["q"], s["k"], s["v"] = _normal(g, T, H, d), _normal(g, T, Hkv, d), _normal(g, T, Hkv, d)
        s["frequencies"] = _frequencies(d, case["scale"])
        s["turns"] = _turns(s["frequencies"])
        b, pos = _positions(s)
        s["positions"] = (pos + case["ahead"]).int()
        if case["norm"]:
            _norm_weights(g, s, d)
        return s
    # weights as attention leaves them: most tokens have little, a few have much, some none at all
    received = torch.exp(2 * torch.randn((pages, Hkv, page), generator=g, device="cuda") - 4)
    received[torch.rand(received.shape, generator=g, device="cuda") < 0.05] = 0
    s["received"] = received
    if case["path"] == "weigh":
        received *= H // Hkv * max(new) / max(lengths)  # as much as these tokens give
        s["q"] = _normal(g, T, H, d)
        s["after"] = torch.zeros_like(received)
        s["lse"] = _log_sums(s)
    else:
        s["to_table"] = to_table
    return s


def _positions(s):
    """The sequence of each new token, and its place there."""
    rows = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["starts"][1:], rows, right=True)
    return b, s["lengths"][b].long() - s["starts"][b + 1].long() + rows


def _pairs(x, r, neighbours):
    """The two values of every pair of the first r."""
    return (x[..., 0:r:2], x[..., 1:r:2]) if neighbours else (x[..., :r // 2], x[..., r // 2:r])


def _joined(u, v, rest, neighbours):
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if neighbours else torch.cat([u, v], -1), rest], -1)


def _rotated(x, cos, sin, neighbours):
    r = 2 * cos.shape[-1]
    u, v = _pairs(x, r, neighbours)
    return _joined(u * cos - v * sin, u * sin + v * cos, x[..., r:], neighbours)


def _angles(s):
    angle = s["positions"].double()[:, None] * s["frequencies"]
    return angle.cos().float()[:, None], angle.sin().float()[:, None]


def _plain_rotated(s, x, cos, sin):
    case, y, w = s["case"], s[x].float(), s[x + "_weight"]
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _rotated(y, cos, sin, case.get("pairs", False)).to(torch.bfloat16)


def _plain_rotate(s):
    angles = _angles(s)
    return {"q": _plain_rotated(s, "q", *angles), "k": _plain_rotated(s, "k", *angles)}


def _plain_gradients(s, x, cos, sin):
    case, w = s["case"], s[x + "_weight"]
    turned = _rotated(s["d" + x + "_out"].float(), cos, -sin, case["pairs"])
    if w is None:
        return {"d" + x: turned.to(torch.bfloat16)}
    y = s[x].float()
    scale = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    unit = y * scale
    weighted = turned * w.float()
    dx = scale * (weighted - unit * (weighted * unit).mean(-1, keepdim=True))
    return {"d" + x: dx.to(torch.bfloat16), "d" + x + "_weight": (turned * unit).double().sum((0, 1)).float()}


def _plain_rotate_bwd(s):
    angles = _angles(s)
    return {**_plain_gradients(s, "q", *angles), **_plain_gradients(s, "k", *angles)}


def _plain_into(s, x, rows, at, slot):
    """Rows of k or v into the cache, and what it then holds of them."""
    pool = s[x + "_pool"]
    if not s["case"]["e4m3"]:
        pool[at, :, slot] = rows
        return pool[at, :, slot]
    e = _row_exponents(rows.float())
    pool.view(torch.uint8)[at, :, slot] = (rows.float() * _power(-e)).to(torch.float8_e4m3fn).view(torch.uint8)
    s[x + "_exp"][at, :, slot] = e.to(torch.int8)
    return (pool.view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float() * _power(s[x + "_exp"][at, :, slot])).to(torch.bfloat16)


def _plain_enter(s):
    page = s["case"]["page"]
    b, pos = _positions(s)
    where = s["table"][b, pos // page].long(), pos % page
    angles = _angles(s)
    return {"q": _plain_rotated(s, "q", *angles), "k": _plain_into(s, "k", _plain_rotated(s, "k", *angles), *where),
            "v": _plain_into(s, "v", s["v"], *where)}


def _scores(s):
    """Scores [B, Hkv, rep, most, reach] of every sequence's new tokens, -inf where a token does not attend a key; rows and positions of the
    tokens [B, most] (those that a sequence has not got repeat its last one), and which there are."""
    case = s["case"]
    B, H, Hkv, d = (case[k] for k in ("B", "H", "Hkv", "d"))
    rep, most, reach = H // Hkv, s["most"], s["reach"]
    keys = s["k_pool"].view(torch.uint8)[s["table"].long()].view(s["k_pool"].dtype).float()
    if case["e4m3"]:
        keys = keys * _power(s["k_exp"][s["table"].long()])
    keys = keys.permute(0, 2, 1, 3, 4).reshape(B, Hkv, reach, d)
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.arange(most, device="cuda").expand(B, most)
    real = i < new[:, None]
    i = torch.minimum(i, new[:, None] - 1)
    rows = s["starts"][:-1, None].long() + i
    pos = (s["lengths"].long() - new)[:, None] + i
    key = torch.arange(reach, device="cuda")
    seen = key <= pos[..., None]
    if case["window"]:
        seen &= (key > pos[..., None] - case["window"]) | (key < case["sinks"])
    q = s["q"].float()[rows].view(B, most, Hkv, rep, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, rep * most, d)
    score = (q @ keys.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(B, Hkv, rep, most, reach)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    return score, rows, real, seen


def _log_sums(s):
    """What attention leaves beside its output: lse [H, T] of the scores."""
    case = s["case"]
    score, rows, real, _ = _scores(s)
    lse = torch.empty((case["H"], s["T"]), device="cuda")
    lse[:, rows] = torch.logsumexp(score, -1).permute(1, 2, 0, 3).reshape(case["H"], case["B"], s["most"])
    return lse


def _plain_weigh(s):
    case = s["case"]
    B, H, Hkv, page = (case[k] for k in ("B", "H", "Hkv", "page"))
    score, rows, real, seen = _scores(s)
    lse = s["lse"][:, rows].view(Hkv, H // Hkv, B, s["most"]).permute(2, 0, 1, 3)
    lse = torch.where(real[:, None, None], lse, torch.full_like(lse, math.inf))  # rows that repeat the last token count for nothing
    weight = score.sub_(lse[..., None]).exp_().sum((2, 3))
    by_pages = (B, Hkv, -1, page)
    weight = weight.view(by_pages).transpose(1, 2)
    at = s["table"].long()
    if case["add"]:
        old = torch.arange(s["reach"], device="cuda") < (s["lengths"] - (s["starts"][1:] - s["starts"][:-1]))[:, None]
        weight = weight + torch.where(old.view(B, -1, 1, page), s["received"][at], torch.zeros((), device="cuda"))
    attended = seen.any(1).view(B, -1, 1, page)
    s["after"][at] = torch.where(attended, weight, s["after"][at])
    return {"received": s["after"]}


def _plain_evict(s):
    case = s["case"]
    B, Hkv, page, d, budget = (case[k] for k in ("B", "Hkv", "page", "d", "budget"))
    at = s["table"].long()
    weight = s["received"][at].permute(0, 2, 1, 3).reshape(B, Hkv, s["reach"])
    place = torch.arange(s["reach"], device="cuda")
    n = s["lengths"].long()[:, None]
    always = (place < case["sinks"]) | (place >= n - case["recent"])
    weight = torch.where(always[:, None], math.inf, weight).masked_fill((place >= n)[:, None], -math.inf)
    keep = min(budget, s["reach"])
    kept = weight.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    left = n.clamp(max=budget)
    there = torch.arange(keep, device="cuda") < left
    kept = kept.masked_fill(~there[:, None], s["reach"]).sort(-1).values
    # rows of the pools [pages, Hkv, page]; places that stay empty move a row of the spare page onto itself
    j = torch.arange(keep, device="cuda").expand(B, keep)
    head = torch.arange(Hkv, device="cuda")[:, None]
    spare = (s["spare"] * Hkv + head) * page + j[:, None] % page
    inside = torch.where(there[:, None], kept, torch.zeros_like(kept))
    source = (at.gather(1, (inside // page).view(B, -1)).view(B, Hkv, keep) * Hkv + head) * page + inside % page
    target_page = s["to_table"].long().gather(1, torch.where(there, j // page, torch.zeros_like(j)))
    target = (target_page[:, None] * Hkv + head) * page + j[:, None] % page
    source, target = torch.where(there[:, None], source, spare).flatten(), torch.where(there[:, None], target, spare).flatten()

    def moved(pool, width):
        rows = pool.view(torch.uint8).view(-1, width)
        rows[target] = rows[source]

    size = 1 if case["e4m3"] else 2
    moved(s["k_pool"], size * d)
    moved(s["v_pool"], size * d)
    moved(s["received"], 4)
    all_kept = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    all_kept[..., :keep] = kept.masked_fill(~there[:, None], -1).int()
    out = {"lengths": left[:, 0].int(), "kept": all_kept, "received": s["received"]}
    if not case["e4m3"]:
        return {**out, "k": s["k_pool"], "v": s["v_pool"]}
    moved(s["k_exp"], 1)
    moved(s["v_exp"], 1)
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), left[:, 0], output_size=s["T"])
    slot = torch.arange(s["T"], device="cuda") - s["starts"].long()[b]
    at, slot = s["to_table"].long()[b, slot // page], slot % page

    def held(x):
        return (s[x + "_pool"].view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float() * _power(s[x + "_exp"][at, :, slot])).to(torch.bfloat16)

    return {**out, "k": held("k"), "v": held("v")}


def _own(s):
    from paper_2309_12307_b200 import binding

    case = s["case"]
    path = case["path"]
    if path in ("rotate", "rotate_bwd"):
        how = dict(positions=s["positions"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS if case["norm"] else None, interleaved=case["pairs"])
        if path == "rotate":
            q, k = binding.s2a_rotate(s["q"], s["k"], s["turns"], **how)
            return {"q": q, "k": k}
        dq, dk, dq_weight, dk_weight = binding.s2a_rotate_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["turns"], **how)
        return {"dq": dq, "dk": dk, **({"dq_weight": dq_weight, "dk_weight": dk_weight} if case["norm"] else {})}
    cache = binding.PagedCache(s["k_pool"], s["v_pool"], s["k_exp"], s["v_exp"])
    where = s["table"], s["starts"], s["lengths"]
    if path == "enter":
        q = binding.s2a_rotate_write(cache, s["q"], s["k"], s["v"], s["turns"], *where, positions=s["positions"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=EPS if case["norm"] else None)
        k, v = binding.s2a_cache_read(cache, *where, tokens=s["T"])
        return {"q": q, "k": k, "v": v}
    if path == "weigh":
        binding.s2a_paged_weights(s["q"], s["lse"], cache, *where, s["after"], before=s["received"] if case["add"] else None, max_new=s["most"],
                                  window=case["window"], sinks=case["sinks"])
        return {"received": s["after"]}
    lengths, kept = binding.s2a_cache_evict(cache, s["received"], s["table"], s["lengths"], s["to_table"], case["budget"], sinks=case["sinks"],
                                            recent=case["recent"])
    out = {"lengths": lengths, "kept": kept, "received": s["received"]}
    if not case["e4m3"]:
        return {**out, "k": s["k_pool"], "v": s["v_pool"]}
    k, v = binding.s2a_cache_read(cache, s["to_table"], s["starts"], lengths, tokens=s["T"])
    return {**out, "k": k, "v": v}


_PLAIN = {"rotate": _plain_rotate, "rotate_bwd": _plain_rotate_bwd, "enter": _plain_enter, "weigh": _plain_weigh, "evict": _plain_evict}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["path"]](state)


def work(case):
    H, Hkv, d, path = case["H"], case["Hkv"], case["d"], case["path"]
    if path in ("rotate", "rotate_bwd"):
        # read and written once; the gradients of norms need what went in as well
        passes = 3 if path == "rotate_bwd" and case["norm"] else 2
        return {"bytes": passes * 2 * case["T"] * (H + Hkv) * d + 4 * case["T"], "flops": 0}
    new, lengths = _sizes(case)
    row = d + 1 if case["e4m3"] else 2 * d  # bytes of a token of a head in the cache
    T = sum(new)
    if path == "enter":
        # q is read and written, k and v are read and written into the cache, which is read and k and v are written
        return {"bytes": 4 * T * H * d + 2 * T * Hkv * (2 * 2 * d + 2 * row) + 4 * T, "flops": 0}
    if path == "evict":
        kept = sum(min(n, case["budget"]) for n in lengths)
        back = 2 * (row + 2 * d) if case["e4m3"] else 0
        return {"bytes": Hkv * (4 * sum(lengths) + kept * (2 * 2 * row + 4 + 4 + back)), "flops": 0}
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
    return {"bytes": keys * Hkv * (row + (8 if case["add"] else 4)) + 2 * T * H * d + 4 * T * H, "flops": 2 * d * H * pairs}


# ---------------------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------------------
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


def _exact_matrix(s):
    """Each position's rotation as complex numbers of size one."""
    case = s["case"]
    r = case.get("r", case["d"])
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    angle = s["positions"].double()[:, None] * (case["scale"] * torch.exp(-2 * i / r * math.log(BASE)))
    return torch.polar(torch.ones_like(angle), angle)[:, None]


def _exact_turned(x, turn, neighbours):
    r, y = 2 * turn.shape[-1], x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if neighbours else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rotation(s):
    case, turn = s["case"], _exact_matrix(s)
    out = {}
    for x in ("q", "k"):
        y, w = s[x].double(), s[x + "_weight"]
        if w is not None:
            y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / case["d"] + EPS) * w.double()
        out[x] = _exact_turned(y, turn, case.get("pairs", False))
    return out


def _exact_gradients(s):
    case, turn = s["case"], _exact_matrix(s).conj()
    out = {}
    for x in ("q", "k"):
        back, w = _exact_turned(s["d" + x + "_out"].double(), turn, case["pairs"]), s[x + "_weight"]
        if w is None:
            out["d" + x] = back
            continue
        y = s[x].double()
        size = torch.sqrt((y ** 2).sum(-1, keepdim=True) / case["d"] + EPS)
        g = back * w.double()
        out["d" + x] = g / size - y * (g * y).sum(-1, keepdim=True) / (case["d"] * size ** 3)
        out["d" + x + "_weight"] = (back * y / size).sum((0, 1))
    return out


def _exact_weigh(s):
    case = s["case"]
    new, lengths = _sizes(case)
    H, Hkv, d, page = (case[k] for k in ("H", "Hkv", "d", "page"))
    out = s["after"].double()
    at = 0
    for b in range(case["B"]):
        n, length = new[b], lengths[b]
        pages = s["table"][b, :-(-length // page)].long()
        query = torch.arange(length - n, length, device="cuda")[:, None]
        keys = torch.arange(length, device="cuda")[None]
        hidden = keys > query
        if case["window"]:
            hidden = hidden | ((query - keys >= case["window"]) & (keys >= case["sinks"]))
        attended = (~hidden).any(0).nonzero()[:, 0]
        for hk in range(Hkv):
            pool = s["k_pool"][pages, hk]
            pool = _exact_values(pool, s["k_exp"][pages, hk]) if case["e4m3"] else pool.double()
            k = pool.reshape(-1, d)[:length]
            weight = torch.zeros(length, dtype=torch.float64, device="cuda")
            if case["add"]:
                weight[:length - n] = s["received"][pages, hk].reshape(-1)[:length - n].double()
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                score = (s["q"][at:at + n, h].double() @ k.T) / math.sqrt(d)
                score[hidden] = -math.inf
                weight += torch.exp(score - s["lse"][h, at:at + n, None].double()).sum(0)
            out[pages[attended // page], hk, attended % page] = weight[attended]
        at += n
    return {"received": out}


def _exact_evict(s):
    case = s["case"]
    _, lengths = _sizes(case)
    B, Hkv, page, budget = (case[k] for k in ("B", "Hkv", "page", "budget"))
    left = [min(n, budget) for n in lengths]
    kept = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    received = s["received"].double()
    pools = {x: s[x + "_pool"].clone() for x in ("k", "v")} if not case["e4m3"] else {x: [] for x in ("k", "v")}
    for b in range(B):
        n, m = lengths[b], left[b]
        place = torch.arange(n, device="cuda")
        page_of = s["table"][b].long()[place // page]
        to_place = torch.arange(m, device="cuda")
        to_page = s["to_table"][b].long()[to_place // page]
        rows = {x: [] for x in ("k", "v")}
        for hk in range(Hkv):
            weight = s["received"][page_of, hk, place % page].double()
            weight[:case["sinks"]] = math.inf
            weight[n - min(n, case["recent"]):] = math.inf
            border = weight.sort().values[n - m]  # the least weight that is kept
            above = weight > border
            ties = ((weight == border).cumsum(0) <= m - above.sum()) & (weight == border)
            mine = (above | ties).nonzero()[:, 0]
            kept[b, hk, :m] = mine.int()
            received[to_page, hk, to_place % page] = s["received"][page_of[mine], hk, mine % page].double()
            for x in ("k", "v"):
                value = s[x + "_pool"].view(torch.uint8)[page_of[mine], hk, mine % page]
                if case["e4m3"]:
                    rows[x].append(_exact_values(value, s[x + "_exp"][page_of[mine], hk, mine % page]))
                else:
                    pools[x].view(torch.uint8)[to_page, hk, to_place % page] = value
        if case["e4m3"]:
            for x in ("k", "v"):
                pools[x].append(torch.stack(rows[x], 1))
    out = {"lengths": torch.tensor(left, dtype=torch.int32, device="cuda"), "kept": kept, "received": received}
    return {**out, **{x: torch.cat(pools[x]) if case["e4m3"] else pools[x] for x in ("k", "v")}}


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "rotate":
        return _exact_rotation(s)
    if path == "rotate_bwd":
        return _exact_gradients(s)
    if path == "weigh":
        return _exact_weigh(s)
    if path == "evict":
        return _exact_evict(s)
    out = {**_exact_rotation(s), "v": s["v"].double()}
    # (the cache holds rotated keys: rounded to bf16, then to its own type)
    out["k"] = out["k"].to(torch.bfloat16)
    return {x: _exact_rounded(out[x]) if case["e4m3"] and x != "q" else out[x].double() for x in ("q", "k", "v")}
