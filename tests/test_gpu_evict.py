"""Weights of cached tokens, and eviction by them, on the GPU against their definitions in 64 bits (oracle/evict_torch.py)."""
import ctypes
import math

import pytest
import torch
from test_gpu_paged import Job

from oracle import evict_torch as ref
from paper_2309_12307_b200 import binding as s2a

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
MARK = -7.0


def weigh(job, lse=None, before=None, in_place=False, scale=None, window=0, sinks=0, max_new=None, q=None, **kw):
    """received before and after one call, lse, and `before`."""
    q = job.q if q is None else q
    scale = 1 / math.sqrt(job.d) if scale is None else scale
    if lse is None:
        _, lse = job.attend(scale=scale, window=window, sinks=sinks)
    shape = job.cache.k.shape[:3]
    if before == "some":
        before = torch.rand(shape, generator=torch.Generator().manual_seed(5)).cuda()
    received = before.clone() if in_place else torch.full(shape, MARK, device="cuda")
    start = received.clone()
    most = max(1, max(n for n, _ in job.sizes)) if max_new is None else max_new
    s2a.s2a_paged_weights(q, lse, job.cache, *job.where, received, before=received if in_place else before, max_new=most, scale=scale, window=window, sinks=sinks, **kw)
    return start, received, lse, before


def check(job, scale=None, window=0, sinks=0, **kw):
    """Entries that no new token attends are left alone.  The others: scores as sums of d products in 32 bits (each addition 2^-24 of a partial sum, at most |q| |k|); their
    difference from lse, both times 1 / ln 2, 2^-23 of either; the exponential 2^-21; sums of all rows 2^-24 for each addition."""
    start, received, lse, before = weigh(job, scale=scale, window=window, sinks=sinks, **kw)
    assert s2a.device_status() == (0, 0)
    scale = 1 / math.sqrt(job.d) if scale is None else scale
    q, host = job.q.cpu(), job.host_cache()
    want, written = ref.paged_weights(q, lse.cpu(), host, job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), start.cpu(), None if before is None else before.cpu(),
                                      scale, window, sinks)
    got = received.cpu()
    assert torch.equal(got[~written], start.cpu()[~written])
    rows = [r for r in range(job.T) if job.rows()[r]]
    if not rows:
        return
    reach = scale * float(q[rows].double().norm(dim=-1).max()) * float(job.all_k.double().norm(dim=-1).max())
    most_lse = float(lse[:, rows].abs().max())
    count = max(n for n, _ in job.sizes) * job.H // job.Hkv
    rel = job.d * 2.0**-24 * reach + (reach + most_lse) * 2.0**-22 + 2.0**-20 + count * 2.0**-24
    assert rel < 0.02  # (the bound says something)
    off = (got[written].double() - want[written]).abs()
    assert (off <= rel * want[written] + 1e-37).all(), float((off / (rel * want[written] + 1e-37)).max())


BATCHES = [[(1, 1)], [(1, 1000)], [(1, 17), (1, 16), (1, 15), (1, 300)], [(0, 0), (3, 50), (0, 40), (1, 1), (33, 33), (2, 700)], [(5, 5)], [(129, 400), (1, 77)],
           [(200, 1111)], [(64, 64), (7, 4000)], [(1, 33), (300, 301), (16, 128), (2, 129)]]


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes", BATCHES)
@pytest.mark.parametrize("H,Hkv,d,page", [(4, 2, 64, 16), (3, 3, 128, 64), (14, 2, 128, 16), (8, 1, 64, 256)])
def test_weights(dtype, sizes, H, Hkv, d, page):
    job = Job(sizes, H=H, Hkv=Hkv, d=d, page=page, dtype=dtype, before=2, after=3, seed=len(sizes))
    check(job, before="some")
    # by itself each row's weights add up to one
    _, alone, _, _ = weigh(job)
    per_head = torch.where(alone == MARK, 0.0, alone).double().sum((0, 2)).cpu()
    rows = sum(n for n, _ in sizes) * H // Hkv
    assert (per_head - rows).abs().max() <= 1e-3 * rows + 1e-9


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (64, 0), (100, 64), (130, 1000), (5000, 5), (300, 17)])
@pytest.mark.parametrize("sizes", [[(1, 1000)], [(0, 9), (3, 50), (1, 1), (2, 700)], [(200, 1111), (1, 600)]])
def test_windows(dtype, window, sinks, sizes):
    job = Job(sizes, H=4, Hkv=2, d=64, page=16, dtype=dtype, after=1)
    check(job, window=window, sinks=sinks, before="some", in_place=True)


def workspace_bytes(job, window, sinks):
    """Bytes with which a call's rows are split over several blocks; 0: they are not."""
    from test_paged_cpu import Batch, Cache

    c = job.cache
    exps = (0, 0) if c.k_exp is None else (c.k_exp.data_ptr(), c.v_exp.data_ptr())
    cache = Cache(k=c.k.data_ptr(), v=c.v.data_ptr(), k_exp=exps[0], v_exp=exps[1], type=int(job.dtype == E4M3), pages=c.k.shape[0], Hkv=job.Hkv, page_size=job.page, d=job.d)
    batch = Batch(table=job.table.data_ptr(), starts=job.starts.data_ptr(), lengths=job.lengths.data_ptr(), width=job.table.shape[1], B=len(job.sizes), T=job.T)
    return s2a.load().s2a_paged_weights_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), job.H, max(n for n, _ in job.sizes), window, sinks)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 17), (100, 300), (300, 17), (300, 300), (300, 0)])
@pytest.mark.parametrize("sizes,H,Hkv", [([(700, 1500)], 8, 1), ([(300, 301), (3, 900), (520, 700)], 14, 2)])
def test_rows_that_are_split(dtype, window, sinks, sizes, H, Hkv):
    """Many rows and few keys: several blocks have the same keys, with a window that leaves each key some of the rows."""
    job = Job(sizes, H=H, Hkv=Hkv, d=64, page=16, dtype=dtype, after=1)
    assert workspace_bytes(job, window, sinks) > 0
    check(job, window=window, sinks=sinks, before="some", in_place=True)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 17)])
def test_a_workspace_that_is_too_small_or_as_large_as_needed(dtype, window, sinks):
    job = Job([(700, 1500)], H=8, Hkv=1, d=64, page=16, dtype=dtype)
    need = workspace_bytes(job, window, sinks)
    for size in (0, 256, need - 1, need):
        check(job, window=window, sinks=sinks, before="some", workspace=torch.full((size,), 255, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_pages_behind_a_window_are_not_needed(dtype):
    job = Job([(2, 700), (150, 900)], H=4, Hkv=2, d=64, page=16, dtype=dtype)
    want, got = [], []
    for out in (want, got):
        _, received, lse, _ = weigh(job, window=40, sinks=20)
        out.append(received)
        job.table[0, 2:(698 - 40) // 16] = -1  # given back
        job.table[1, 2:(750 - 40) // 16] = 10**6
    assert torch.equal(want[0], got[0]) and s2a.device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("in_place", [False, True])
def test_added_to_what_was(dtype, in_place):
    check(Job([(3, 50), (1, 200), (70, 70)], H=8, Hkv=2, d=128, page=32, dtype=dtype), before="some", in_place=in_place)


def test_weights_add_up_over_calls():
    """Token by token and all at once."""
    one = Job([(40, 40)], H=4, Hkv=2, d=64, page=16)
    _, whole, lse, _ = weigh(one)
    total = torch.full_like(whole, math.nan)  # pages are not cleared
    for i in range(40):
        starts, lengths = torch.tensor([i, i + 1], dtype=torch.int32).cuda(), torch.tensor([i + 1], dtype=torch.int32).cuda()
        s2a.s2a_paged_weights(one.q, lse, one.cache, one.table, starts, lengths, total, before=total, max_new=1)
    mine = whole != MARK
    assert torch.equal(mine, ~torch.isnan(total))
    assert torch.allclose(whole[mine], total[mine], rtol=2.0**-17, atol=0)  # 80 additions of 2^-24, and scores as above


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("scale", [2.0**-20, 4.0])
def test_scales(dtype, scale):
    check(Job([(3, 50), (70, 200)], H=4, Hkv=2, d=64, page=16, dtype=dtype, normal=1.0 if scale < 1 else 0.25), scale=scale)


@pytest.mark.parametrize("by", [2.0**-60, 2.0**60])
def test_large_and_small_keys_and_queries(by):
    """Keys far from one and queries by as much the other way: scores as ever."""
    for dtype in (BF16, E4M3):
        job = Job([(3, 50), (20, 100)], H=4, Hkv=2, d=64, page=16, dtype=dtype, normal=by)
        job.q = (job.q.float() / by).to(BF16)
        check(job)


@pytest.mark.parametrize("new", [1, 10, 30, 200])  # (of two rows each: 1 and 10 are the streaming kernel's)
@pytest.mark.parametrize("q_power,k_power", [(-100, 100), (-112, 112), (100, -117), (120, -126), (-118, 118), (0, -120), (-120, 0)])
def test_queries_and_keys_at_the_ends_of_the_range(q_power, k_power, new):
    """8-bit keys whose powers of two and those of the queries cancel, or leave next to nothing."""
    for window, sinks in ((0, 0), (70, 3)):
        job = Job([(new, 300)], H=4, Hkv=2, d=64, page=32, dtype=E4M3)
        job.all_k *= 2.0**k_power
        s2a.s2a_cache_write(job.cache, job.all_k, job.all_v, job.table, job.all_starts, job.lengths)
        job.q *= 2.0**q_power
        check(job, window=window, sinks=sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 10, 200])
def test_scores_that_are_zero_between_the_largest_numbers(d, new):
    """Queries and keys near 2^127 with nothing in common: the scores are zero, whatever power of two they would be multiplied with, and each weight is exp(-lse)."""
    job = Job([(new, 300)], H=4, Hkv=2, d=d, page=32, dtype=E4M3)
    job.all_k[..., :d // 2] = 0
    job.all_k[..., d // 2:] = 2.0**127
    job.q[..., d // 2:] = 0
    job.q[..., :d // 2] = 2.0**127
    s2a.s2a_cache_write(job.cache, job.all_k, job.all_v, job.table, job.all_starts, job.lengths)
    start, received, lse, _ = weigh(job)
    want, written = ref.paged_weights(job.q.cpu(), lse.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), start.cpu(), None, d**-0.5)
    # lse (at most log 300) times 1 / ln 2, the exponential, and sums of 2 * new rows: as in check(), without scores
    rel = 6 * 2.0**-22 + 2.0**-20 + 2 * new * 2.0**-24
    off = (received.cpu()[written].double() - want[written]).abs()
    assert (off <= rel * want[written]).all() and s2a.device_status() == (0, 0)


@pytest.mark.parametrize("new", [2, 16, 40])
def test_rows_of_one_call_far_from_one_another(new):
    """Keys near 2^118.  Every other row of q is as large and has nothing in common with them, the others are as small: their scores are ordinary."""
    d = 64
    job = Job([(new, 300)], H=2, Hkv=1, d=d, page=32, dtype=E4M3)
    job.all_k[..., :d // 2] = 0
    job.all_k *= 2.0**118
    s2a.s2a_cache_write(job.cache, job.all_k, job.all_v, job.table, job.all_starts, job.lengths)
    job.q[::2, :, d // 2:] = 0
    job.q[::2] *= 2.0**118
    job.q[1::2] *= 2.0**-118
    i = torch.arange(300 - new, 300)
    host = job.host_cache()
    from oracle.paged_torch import sequence_values
    s = d**-0.5 * torch.einsum("thc,jc->htj", job.q.cpu().double(), sequence_values(host, "k", job.table.cpu(), 0, 300)[0])
    lse = s.masked_fill(~ref.attends(i, 300, 0, 0), -math.inf).logsumexp(-1).float().cuda()  # (what is looked at here are the weights)
    start, received, _, _ = weigh(job, lse=lse)
    want, written = ref.paged_weights(job.q.cpu(), lse.cpu(), host, job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), start.cpu(), None, d**-0.5)
    reach = d**-0.5 * float((job.q.cpu()[1::2].double() * 2.0**118).norm(dim=-1).max()) * float((job.all_k.double() * 2.0**-118).norm(dim=-1).max())
    rel = d * 2.0**-24 * reach + (reach + float(lse.abs().max())) * 2.0**-22 + 2.0**-20 + 2 * new * 2.0**-24
    off = (received.cpu()[written].double() - want[written]).abs()
    assert rel < 0.02 and (off <= rel * want[written]).all() and s2a.device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_what_is_not_attended_does_not_matter(dtype):
    """Keys that some rows do not attend: NaN there reaches no other key's weight."""
    job = Job([(5, 40), (90, 140)], H=4, Hkv=2, d=64, page=16, dtype=dtype)
    _, want, lse, _ = weigh(job)
    bad = job.all_k.clone()
    bad[39], bad[40 + 139] = math.nan, math.inf  # each sequence's last token
    s2a.s2a_cache_write(job.cache, bad, job.all_v, job.table, job.all_starts, job.lengths)
    _, got, _, _ = weigh(job, lse=lse)
    keep = torch.ones_like(want, dtype=torch.bool)
    for b, j in ((0, 39), (1, 139)):
        keep[int(job.table[b, j // 16]), :, j % 16] = False
    assert torch.equal(want[keep], got[keep]) and not torch.isfinite(got[~keep]).any()


@pytest.mark.parametrize("n", [1, 3, 40])
def test_a_score_of_minus_infinity_is_a_weight_of_zero(n):
    job = Job([(n, 60)], H=4, Hkv=2, d=64, page=16)
    _, clean, lse, _ = weigh(job)
    job.q[..., 5] = job.q[..., 5].abs() + 0.5
    k = job.all_k.clone()
    k[7, :, 5] = -math.inf
    s2a.s2a_cache_write(job.cache, k, job.all_v, job.table, job.all_starts, job.lengths)
    _, received, lse, _ = weigh(job, lse=lse)
    at = int(job.table[0, 0]), slice(None), 7
    assert (received[at] == 0).all() and torch.isfinite(received).all()


def test_many_query_heads_of_a_kv_head():
    """More rows a token than the streaming kernel takes."""
    check(Job([(1, 300), (2, 90), (0, 5)], H=64, Hkv=1, d=64, page=16), before="some")
    check(Job([(1, 1000)], H=64, Hkv=1, d=128, page=64, dtype=E4M3))


def test_the_same_twice_on_another_stream_and_captured():
    job = Job([(1, 300), (90, 400), (3, 1000)], H=8, Hkv=2, d=128, page=32)
    _, want, lse, before = weigh(job, before="some")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    _, again, _, _ = weigh(job, lse=lse, before=before, stream=stream)
    stream.synchronize()
    assert torch.equal(want, again)
    out = torch.full_like(want, MARK)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2a.s2a_paged_weights(job.q, lse, job.cache, *job.where, out, before=before, max_new=90)
    graph.replay()
    assert torch.equal(want, out)
    job.lengths -= 1
    graph.replay()
    _, lse_now = job.attend()
    lse.copy_(lse_now)
    out.fill_(MARK)
    graph.replay()
    _, want, _, _ = weigh(job, lse=lse, before=before)
    assert torch.equal(want, out) and s2a.device_status() == (0, 0)


def test_bad_batches_are_reported():
    job = Job([(3, 50), (2, 20)], H=4, Hkv=2, d=64, page=16)
    _, lse = job.attend()
    received = torch.full(job.cache.k.shape[:3], MARK, device="cuda")
    for bad, where in ((1003, (job.table.clamp(max=0) - 1, job.starts, job.lengths)), (1002, (job.table, job.starts, job.lengths * 0)),
                       (1001, (job.table, job.starts + 1, job.lengths)), (1004, job.where)):
        s2a.s2a_paged_weights(job.q, lse, job.cache, *where, received, max_new=2 if bad == 1004 else 3)
        torch.cuda.synchronize()
        with pytest.raises(s2a.S2AError):
            s2a.s2a_paged_weights(job.q, lse, job.cache, *job.where, received)
        assert s2a.device_status() == (s2a.S2A_ERR_BAD_INDEX, bad) and s2a.device_status() == (0, 0)


# ---------------------------------------------------------------------------------------------- eviction
def evicted(sizes, budget, sinks, recent, Hkv=2, d=64, page=16, dtype=BF16, received=None, seed=0, wider=0, share=False):
    """One eviction of a batch of sequences of these lengths, checked: what is kept, what the new pages hold, and that nothing else changes."""
    job = Job([(0, n) for n in sizes], H=Hkv, Hkv=Hkv, d=d, page=page, dtype=dtype, seed=seed)
    cache, B = job.cache, len(sizes)
    table = job.table.clone()
    if share:
        table[1] = table[0]
    need = [-(-min(n, budget) // page) for n in sizes]
    pages, extra = cache.k.shape[0], sum(need) + 1
    more = s2a.PagedCache(*(None if x is None else torch.cat((x, torch.full((extra, *x.shape[1:]), 0, dtype=torch.uint8, device="cuda").view(x.dtype) if x.dtype != BF16 else
                                                                        torch.zeros((extra, *x.shape[1:]), dtype=BF16, device="cuda"))) for x in (cache.k, cache.v, cache.k_exp, cache.v_exp)))
    g = torch.Generator().manual_seed(seed + 1)
    order = (torch.randperm(extra, generator=g) + pages).tolist()
    to_table = torch.full((B, max(1, max(need)) + wider), -5, dtype=torch.int32)
    for b, n in enumerate(need):
        to_table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    if received is None:
        received = torch.randn((pages, Hkv, page), generator=g).exp()
    received = torch.cat((received, torch.full((extra, Hkv, page), MARK))).cuda()
    start = {x: None if getattr(more, x) is None else getattr(more, x).clone() for x in ("k", "v", "k_exp", "v_exp")}
    start["received"] = received.clone()
    lengths, kept = s2a.s2a_cache_evict(more, received, table, job.lengths, to_table.cuda(), budget, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    assert s2a.device_status() == (0, 0)
    assert lengths.tolist() == [min(n, budget) for n in sizes]
    want = ref.evict(start["received"].cpu(), table.cpu(), sizes, page, budget, sinks, recent)
    changed = torch.zeros((pages + extra, Hkv, page), dtype=torch.bool)
    now = {x: getattr(more, x).cpu() for x in ("k", "v", "k_exp", "v_exp") if getattr(more, x) is not None}
    now["received"] = received.cpu()
    old = {x: t.cpu() for x, t in start.items() if t is not None}
    for b in range(B):
        for hk in range(Hkv):
            mine = want[b][hk]
            assert kept[b, hk].tolist() == mine + [-1] * (budget - len(mine))
            if not mine:
                continue
            j = torch.tensor(mine)
            source = table[b].cpu().long()[j // page], j % page
            place = torch.arange(len(mine))
            target = to_table[b].long()[place // page], place % page
            changed[target[0], hk, target[1]] = True
            for x in now:
                a, c = now[x][target[0], hk, target[1]], old[x][source[0], hk, source[1]]
                assert torch.equal(a.contiguous().view(torch.uint8), c.contiguous().view(torch.uint8)), x
    for x in now:
        a, c = (t.contiguous().view(torch.uint8).view(*changed.shape, -1) for t in (now[x], old[x]))
        assert torch.equal(a[~changed], c[~changed]), x
    return job, more, received, lengths, kept, to_table.cuda()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hkv,d,page", [(2, 64, 16), (3, 128, 64), (1, 128, 256), (8, 64, 128)])
@pytest.mark.parametrize("sizes,budget,sinks,recent", [([1], 1, 0, 0), ([2, 1, 0, 17], 1, 0, 1), ([1000, 16, 33, 64], 33, 4, 8), ([2100], 1024, 0, 0), ([300, 5000], 64, 64, 0),
                                                       ([129, 128, 127], 128, 1, 120), ([700], 10, 4, 6), ([0, 0], 5, 0, 0), ([40, 50], 1000, 10, 20), ([1025, 3000], 1000, 3, 900)])
def test_the_heaviest_stay_in_order(dtype, Hkv, d, page, sizes, budget, sinks, recent):
    evicted(sizes, budget, sinks, recent, Hkv=Hkv, d=d, page=page, dtype=dtype, wider=1)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "special", "close", "falling"])
@pytest.mark.parametrize("budget", [1, 50, 777])
def test_weights_that_are_equal_or_no_numbers(kind, budget):
    g = torch.Generator().manual_seed(3)
    n, pages = 1500, -(-1500 // 16) + 2
    shape = (pages, 2, 16)
    if kind == "equal":
        w = torch.full(shape, 0.25)
    elif kind == "few":
        w = torch.randint(0, 3, shape, generator=g).float()
    elif kind == "zeros":
        w = torch.where(torch.rand(shape, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0))
    elif kind == "special":
        values = torch.tensor([math.nan, -math.nan, math.inf, -math.inf, 0.0, -0.0, 1.0, -1.0, 1e-45, 3e38])
        w = values[torch.randint(0, len(values), shape, generator=g)]
    elif kind == "close":  # neighbours in the last digits
        w = (torch.tensor(1.0).view(torch.int32) + torch.randint(0, 600, shape, generator=g).int()).view(torch.float32)
    else:
        w = 1.0 / (1 + torch.arange(math.prod(shape)).float().view(shape))
    evicted([n], budget, 0, 0, received=w)
    if budget > 20:
        evicted([n], budget, 4, 16, received=w)


def test_a_budget_that_is_too_large_takes_no_memory():
    job = Job([(0, 20)], H=1, Hkv=1, d=64, page=16)
    received = torch.zeros(job.cache.k.shape[:3], device="cuda")
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    for budget in (2**30, 2**31 - 1):
        with pytest.raises(s2a.S2AError) as e:
            s2a.s2a_cache_evict(job.cache, received, job.table, job.lengths, job.table, budget)
        assert e.value.status == s2a.S2A_ERR_UNSUPPORTED
    assert torch.cuda.max_memory_allocated() - held < 2**20 and s2a.device_status() == (0, 0)


def test_long_sequences():
    evicted([100_003], 4097, 4, 1024, Hkv=1, d=64, page=128, dtype=E4M3)
    evicted([60_000, 58_000, 9, 20_000], 300, 0, 7, Hkv=2, d=64, page=16)
    evicted([420_001], 1000, 4, 100, Hkv=1, d=64, page=256, dtype=E4M3)  # more than a cluster's shared memory holds


def test_old_pages_may_be_shared():
    evicted([200, 180], 60, 4, 20, share=True)


def test_eviction_captured_and_on_another_stream():
    job, cache, received, lengths, kept, to_table = evicted([500, 300], 100, 4, 30)
    n, out = torch.zeros_like(lengths), torch.zeros_like(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2a.s2a_cache_evict(cache, received, job.table, job.lengths, to_table, 100, sinks=4, recent=30, new_lengths=n, kept=out)
    graph.replay()
    assert torch.equal(n, lengths) and torch.equal(out, kept)
    received[job.table.long().flatten()[0]] = 100.0
    graph.replay()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    lengths, kept = s2a.s2a_cache_evict(cache, received, job.table, job.lengths, to_table, 100, sinks=4, recent=30, stream=stream)
    stream.synchronize()
    assert torch.equal(n, lengths) and torch.equal(out, kept) and s2a.device_status() == (0, 0)


def test_bad_tables_are_reported_and_not_followed():
    job, cache, received, _, kept, to_table = evicted([500, 300], 100, 4, 30)
    before = [x.clone() for x in (cache.k, cache.v, received)]
    for bad, args in ((1003, (job.table.clamp(max=0) - 1, job.lengths, to_table)), (1003, (job.table, job.lengths, to_table + 10**6)),
                      (1002, (job.table, job.lengths + 10**6, to_table)), (1002, (job.table, job.lengths * 0 - 1, to_table))):
        s2a.s2a_cache_evict(cache, received, *args, 100, sinks=4, recent=30)
        torch.cuda.synchronize()
        with pytest.raises(s2a.S2AError):
            s2a.s2a_cache_evict(cache, received, job.table, job.lengths, to_table, 100)
        assert s2a.device_status() == (s2a.S2A_ERR_BAD_INDEX, bad) and s2a.device_status() == (0, 0)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (cache.k, cache.v, received)))


# ---------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_a_sequence_served_beyond_its_cache(dtype):
    """A prompt, then single tokens, with the cache cut down whenever it is full: every step's attention against the definition over the tokens that stayed."""
    from oracle import paged_torch, rotate_torch

    g = torch.Generator().manual_seed(11)
    H, Hkv, d, page, budget, most = 4, 2, 64, 16, 48, 80
    turns = s2a.rotary_turns(d, scale=0.25)
    freq = [0.25 * 10000.0 ** (-2 * i / d) for i in range(d // 2)]
    cache = s2a.PagedCache.empty(16, Hkv, page, d, dtype)
    received = torch.full((16, Hkv, page), math.nan, device="cuda")
    tables = [torch.arange(0, 8, dtype=torch.int32).view(1, 8).cuda(), torch.arange(8, 16, dtype=torch.int32).view(1, 8).cuda()]
    held, position, evictions = 0, 0, 0
    for step in range(90):  # full (80 tokens) before step 44, and 32 steps later again
        n = 37 if step == 0 else 1
        q, k, v = (torch.randn(n, h, d, generator=g).to(BF16).cuda() for h in (H, Hkv, Hkv))
        positions = torch.arange(position, position + n, dtype=torch.int32)
        position += n
        if held + n > most:
            lengths = torch.tensor([held], dtype=torch.int32).cuda()
            weights = ref.evict(received.cpu(), tables[0].cpu(), [held], page, budget, 4, 16)[0]
            new_lengths, kept = s2a.s2a_cache_evict(cache, received, tables[0], lengths, tables[1], budget, sinks=4, recent=16)
            assert new_lengths.tolist() == [budget] and kept[0].tolist() == weights
            tables, held, evictions = tables[::-1], budget, evictions + 1
        held += n
        where = tables[0], torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([held], dtype=torch.int32).cuda()
        q_out = s2a.s2a_rotate_write(cache, q, k, v, turns, *where, positions=positions.cuda())
        o, lse = s2a.s2a_paged_fwd(q_out, cache, *where)
        s2a.s2a_paged_weights(q_out, lse, cache, *where, received, before=received)
        want = rotate_torch.rotate(q.cpu(), positions, freq)
        assert ((q_out.cpu().double() - want).abs() <= 2.0**-8 * want.abs() + 2.0**-16 * 8).all()
        host = {"k": cache.k.cpu() if dtype == BF16 else cache.k.view(torch.uint8).cpu(), "v": cache.v.cpu() if dtype == BF16 else cache.v.view(torch.uint8).cpu()}
        if dtype == E4M3:
            host |= {"k_exp": cache.k_exp.cpu(), "v_exp": cache.v_exp.cpu()}
        o_want, lse_want, _, _ = paged_torch.paged_fwd(q_out.cpu(), host, *(x.cpu() for x in where), 1 / math.sqrt(d), 0, 0)
        assert (lse.cpu().double() - lse_want).abs().max() <= 1e-4
        total = torch.cat([received[tables[0][0, j // page].long(), :, j % page][:, None] for j in range(held)], 1).double().cpu()
        assert torch.isfinite(total).all()
    assert evictions == 2 and s2a.device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_pages_past_32_bits(dtype):
    """The same tokens in the last pages of a large pool and in a small one."""
    d, page, n = 128, 256, 600
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, h, d, generator=g).to(BF16).cuda() for h in (2, 1, 1))
    turns, results = s2a.rotary_turns(d), []
    for pages in (8, 2**31 // (page * d) + 8 if dtype == BF16 else 2**32 // (page * d) + 8):
        cache = s2a.PagedCache.empty(pages, 1, page, d, dtype)
        received = torch.zeros((pages, 1, page), device="cuda")
        table, to_table = (torch.tensor([[pages - 1 - i for i in x]], dtype=torch.int32).cuda() for x in ((0, 2, 4), (5, 3)))
        where = table, torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
        q_out = s2a.s2a_rotate_write(cache, q, k, v, turns, *where)
        _, lse = s2a.s2a_paged_fwd(q_out, cache, *where)
        s2a.s2a_paged_weights(q_out, lse, cache, *where, received)
        for few in (1, 7):  # the other kernel
            last = table, torch.tensor([0, few], dtype=torch.int32).cuda(), where[2]
            s2a.s2a_paged_weights(q_out[-few:], lse[:, -few:].contiguous(), cache, *last, received, before=received)
        lengths, kept = s2a.s2a_cache_evict(cache, received, table, where[2], to_table, 400, sinks=3, recent=50)
        back = s2a.s2a_cache_read(cache, to_table, torch.tensor([0, 400], dtype=torch.int32).cuda(), lengths, tokens=400)
        results.append((q_out, kept, *back, received[to_table[0].long()]))
        assert s2a.device_status() == (0, 0)
    assert all(torch.equal(a, b) for a, b in zip(*results))


# ---------------------------------------------------------------------------------------------- refusals
def test_refusals():
    job = Job([(3, 50), (2, 20)], H=4, Hkv=2, d=64, page=16)
    lse, received = torch.zeros((4, job.T), device="cuda"), torch.zeros(job.cache.k.shape[:3], device="cuda")
    to_table = job.table.clone()

    def weights(q=job.q, lse=lse, received=received, before=None, **kw):
        return lambda: s2a.s2a_paged_weights(q, lse, job.cache, *job.where, received, before=before, **kw)

    def evict(received=received, table=job.table, lengths=job.lengths, to_table=to_table, budget=10, **kw):
        return lambda: s2a.s2a_cache_evict(job.cache, received, table, lengths, to_table, budget, **kw)

    for message, call in [("q must have dtype", weights(q=job.q.float())), ("lse must have shape", weights(lse=lse.T.contiguous())), ("received must be a torch.Tensor", weights(received=None)),
                          ("received must have dtype", weights(received=received.half())), ("before must have shape", weights(before=received[:2])),
                          ("before must be a CUDA", weights(before=received.cpu())), ("received must have shape", evict(received=received[0])),
                          ("to_table must be", evict(to_table=to_table[:1])), ("to_table must have dtype", evict(to_table=to_table.long())), ("lengths must have shape", evict(lengths=job.starts)),
                          ("table must be", evict(table=job.table[0])), ("new_lengths must have dtype", evict(new_lengths=job.lengths.long())),
                          ("kept must have shape", evict(kept=torch.zeros((2, 2, 9), dtype=torch.int32, device="cuda")))]:
        with pytest.raises(ValueError, match=message):
            call()
    for call in (weights(max_new=0), weights(max_new=6), weights(window=-1), weights(sinks=-1), weights(scale=0.0), weights(scale=math.nan), weights(q=job.q[:, :3].contiguous(), lse=lse[:3]),
                 evict(budget=0), evict(budget=-1), evict(sinks=6, recent=5), evict(sinks=-1), evict(recent=-1), evict(new_lengths=job.lengths),
                 evict(budget=17, to_table=to_table[:, :1].contiguous()), evict(budget=2**40)):
        with pytest.raises(s2a.S2AError) as e:
            call()
        assert e.value.status == s2a.S2A_ERR_INVALID_ARG
    assert s2a.device_status() == (0, 0)
