"""The paged cache on the GPU against its definition in 64 bits (oracle/paged_torch.py)."""
import math

import pytest
import torch

from oracle import paged_torch as ref
from paper_2309_12307_b200 import binding as s2a

pytestmark = pytest.mark.gpu
BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


class Job:
    """A batch with its cache.  `sizes`: (new tokens, length) of every sequence; `before`, `after`: rows of no sequence.  What the
    sequences do not hold is NaN (in 8 bits: rows marked as NaN), and so are the rows of no sequence."""

    def __init__(self, sizes, H=4, Hkv=2, d=64, page=16, dtype=BF16, before=0, after=0, seed=0, wider=0, normal=1.0):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.H, self.Hkv, self.d, self.page, self.dtype = sizes, H, Hkv, d, page, dtype
        B = len(sizes)
        starts = [before]
        for n, _ in sizes:
            starts.append(starts[-1] + n)
        self.T = starts[-1] + after
        need = [-(-length // page) for _, length in sizes]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=g).tolist()
        table = torch.full((B, max(1, max(need)) + wider), -1, dtype=torch.int32)
        for b, n in enumerate(need):
            table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        self.table, self.starts, self.lengths = (x.cuda() for x in (table, torch.tensor(starts, dtype=torch.int32),
                                                                     torch.tensor([length for _, length in sizes], dtype=torch.int32)))
        self.cache = s2a.PagedCache.empty(pages, Hkv, page, d, dtype)
        for pool in (self.cache.k, self.cache.v):
            pool.view(torch.uint8).fill_(255)  # NaN in either type
        if dtype == E4M3:
            self.cache.k_exp.fill_(ref.NOT_FINITE), self.cache.v_exp.fill_(ref.NOT_FINITE)
        # every token of the sequences, written as one batch of new tokens
        all_starts = [0]
        for _, length in sizes:
            all_starts.append(all_starts[-1] + length)
        self.all_starts = torch.tensor(all_starts, dtype=torch.int32).cuda()
        self.all_k, self.all_v = ((torch.randn(max(1, all_starts[-1]), Hkv, d, generator=g) * normal).to(BF16).cuda() for _ in range(2))
        s2a.s2a_cache_write(self.cache, self.all_k, self.all_v, self.table, self.all_starts, self.lengths)
        self.q = torch.randn(self.T, H, d, generator=g).to(BF16)
        self.q[:before] = math.nan
        self.q[starts[-1]:] = math.nan
        self.q = self.q.cuda()

    @property
    def where(self):
        return self.table, self.starts, self.lengths

    def host_cache(self):
        out = {}
        for x in ("k", "v"):
            pool = getattr(self.cache, x)
            out[x] = pool.view(torch.uint8).cpu() if self.dtype == E4M3 else pool.cpu()
            if self.dtype == E4M3:
                out[x + "_exp"] = getattr(self.cache, x + "_exp").cpu()
        return out

    def rows(self):
        """Rows that belong to a sequence."""
        inside = torch.zeros(self.T, dtype=torch.bool)
        inside[int(self.starts[0]):int(self.starts[-1])] = True
        return inside

    def attend(self, **kw):
        kw.setdefault("max_new", max(1, max(n for n, _ in self.sizes)))
        return s2a.s2a_paged_fwd(self.q, self.cache, *self.where, **kw)

    def check(self, scale=None, window=0, sinks=0, **kw):
        scale = 1 / math.sqrt(self.d) if scale is None else scale
        mark = torch.full((self.T, self.H, self.d), 7.0, dtype=BF16, device="cuda")
        o, lse = self.attend(scale=scale, window=window, sinks=sinks, o=mark, lse=torch.full((self.H, self.T), 7.0, device="cuda"), **kw)
        torch.cuda.synchronize()
        assert s2a.device_status() == (0, 0)
        want, want_lse, size, largest = ref.paged_fwd(self.q.cpu(), self.host_cache(), self.table.cpu(), self.starts.cpu(), self.lengths.cpu(), scale, window, sinks)
        compare(o.cpu(), lse.cpu(), want, want_lse, size, largest, self.rows(), max(length for _, length in self.sizes), self.d, scale,
                float(self.q.cpu()[self.rows()].double().norm(dim=-1).max()) if self.rows().any() else 0.0, self.all_k)


def compare(o, lse, want, want_lse, size, largest, inside, longest, d, scale, q_norm, k):
    """Rows of no sequence untouched; the others as near as the roundings allow: weights and results to bf16 (half a step, 2^-8, each),
    scores as sums of d products in 32 bits (each addition 2^-24 of a partial sum, that at most |q| |k|), sums over the keys likewise.

    Over a cache in 8 bits the weights are fp16 numbers, 2^7 as large relative to 2^r, where r is at most the largest log2(weight) + e of a block of
    128 keys and 2^e the largest power of two of v there (`largest` = 2^r with normalised weights).  Below 2^-14 the step of fp16 is 2^-24, so each
    weight, times 2^-e of its block, is off by up to 2^-25 * 2^-7 * 2^r; v times 2^-e is at most 448, and there are at most `longest` of them."""
    assert (o[~inside] == 7).all() and (lse[:, ~inside] == 7).all()
    o, want, size = o[inside].double(), want[inside], size[inside]
    score = d * 2.0**-24 * scale * q_norm * float(k.double().norm(dim=-1).max()) + 2.0**-20
    slack = longest * 2.0**-24
    off = (o - want).abs()
    allowed = (2.0**-8 + 2 * score + slack) * size + 2.0**-8 * (want.abs() + 2.0**-8 * size) + 1e-30
    allowed += 2.0**-32 * 448 * longest * largest[inside][..., None]
    assert (off <= allowed).all(), float((off / allowed).max())
    off = (lse[:, inside].double() - want_lse[:, inside]).abs()
    assert (off <= score + slack + want_lse[:, inside].abs() * 2.0**-22).all(), float(off.max())


# ---------------------------------------------------------------------------------------------- writing and reading
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("Hkv,d,page", [(1, 64, 16), (2, 128, 16), (5, 64, 64), (8, 128, 128), (40, 128, 32), (3, 128, 256)])
def test_written_tokens_come_back_and_nothing_else_changes(dtype, Hkv, d, page):
    job = Job([(3, 50), (0, 0), (1, 1), (0, 17), (33, 33), (page, 3 * page), (1, page + 1)], Hkv=Hkv, H=Hkv, d=d, page=page, dtype=dtype, before=2, after=3)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(job.T, Hkv, d, generator=g).to(BF16) for _ in range(2))
    k[4] *= 2.0**-128  # subnormal numbers
    v[5] *= 2.0**119
    v[6] = 0
    k[7] = 3.5  # 448 * 2^-7
    before = job.host_cache()
    s2a.s2a_cache_write(job.cache, k.cuda(), v.cuda(), *job.where)
    out = [torch.full((job.T, Hkv, d), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    back = s2a.s2a_cache_read(job.cache, *job.where, k=out[0], v=out[1])
    assert back[0] is out[0] and back[1] is out[1]
    after = job.host_cache()
    assert s2a.device_status() == (0, 0)
    starts, table = job.starts.tolist(), job.table.cpu()
    new = torch.zeros(after["k"].shape[:3], dtype=torch.bool)
    inside = job.rows()
    for x, rows, got in (("k", k, back[0].cpu()), ("v", v, back[1].cpu())):
        assert (got[~inside] == 7).all()
        for b, (n, length) in enumerate(job.sizes):
            for i in range(n):
                pos = length - n + i
                at = int(table[b, pos // page]), slice(None), pos % page
                new[at] = True
                for hk in range(Hkv):
                    row = rows[starts[b] + i, hk]
                    cell = after[x][at[0], hk, at[2]]
                    if dtype == BF16:
                        assert torch.equal(cell, row) and torch.equal(got[starts[b] + i, hk], row)
                    else:
                        codes, e = ref.quantised_row(row)
                        assert torch.equal(cell, codes) and int(after[x + "_exp"][at[0], hk, at[2]]) == e
                        assert torch.equal(got[starts[b] + i, hk].double(), ref.code_values()[codes.long()] * math.ldexp(1.0, e))
    for x in after:
        changed = (after[x].view(torch.uint8) != before[x].view(torch.uint8)) if after[x].dim() == 3 else (after[x].view(torch.uint8) != before[x].view(torch.uint8)).any(-1)
        assert not (changed & ~new).any(), x


def test_every_finite_bf16_number_is_rounded_to_the_nearest_code():
    every = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF16)
    every = every[torch.isfinite(every.float())]
    size = every.float().abs()
    # rows of one magnitude keep all their bits in reach, rows of random ones have values far below the largest
    order = torch.argsort(size)
    rows = torch.cat((every[order], every[torch.randperm(len(every), generator=torch.Generator().manual_seed(0))]))
    rows = rows[:len(rows) // 64 * 64].view(-1, 1, 64)
    T = len(rows)
    cache = s2a.PagedCache.empty(-(-T // 16), 1, 16, 64, E4M3)
    table = torch.arange(cache.k.shape[0], dtype=torch.int32, device="cuda")[None]
    starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, T], [T]))
    s2a.s2a_cache_write(cache, rows.cuda(), rows.cuda(), table, starts, lengths)
    k, v = s2a.s2a_cache_read(cache, table, starts, lengths, tokens=T)
    codes, e = cache.k.view(torch.uint8).cpu().view(-1, 64), cache.k_exp.cpu().view(-1)
    assert torch.equal(k, v) and torch.isfinite(k.float()).all()
    for t in range(T):
        want, want_e = ref.quantised_row(rows[t, 0])
        assert int(e[t]) == want_e and torch.equal(codes[t], want), t
    # what these codes stand for are bf16 numbers
    values = ref.code_values()[codes[:T].long()] * torch.exp2(e[:T].double())[:, None]
    assert torch.equal(k.cpu()[:, 0].double(), values)


def test_a_row_that_is_not_finite_reads_back_as_nan():
    job = Job([(6, 20)], Hkv=2, H=2, d=64, dtype=E4M3)
    k = torch.randn(6, 2, 64).to(BF16)
    k[1, 0, 5], k[2, 1, 0], k[3, 0, 63] = math.inf, math.nan, -math.inf
    s2a.s2a_cache_write(job.cache, k.cuda(), k.cuda(), *job.where)
    got, _ = s2a.s2a_cache_read(job.cache, *job.where, tokens=6)
    bad = torch.zeros(6, 2, dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = bad[3, 0] = True
    nan = torch.isnan(got.cpu().float())
    assert nan[bad].all() and not nan[~bad].any() and s2a.device_status() == (0, 0)


# ---------------------------------------------------------------------------------------------- attention
FORMS = [  # (H, Hkv, d, page)
    (4, 4, 64, 16), (4, 2, 128, 16), (8, 1, 64, 64), (6, 2, 128, 128), (5, 5, 64, 32), (14, 2, 128, 256), (16, 1, 128, 16), (20, 1, 64, 16), (40, 1, 128, 64),
]
SINGLE = [(1, 1), (1, 2), (1, 15), (1, 16), (1, 17), (1, 31), (0, 40), (1, 64), (1, 127), (1, 128), (1, 129), (1, 300), (0, 0)]
DRAFTS = [(2, 2), (4, 100), (3, 129), (1, 260), (0, 9), (4, 17), (2, 128)]
PIECES = [(1, 5), (130, 130), (17, 300), (128, 256), (129, 140), (0, 70), (257, 400), (64, 64), (1, 333)]


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes", [SINGLE, DRAFTS, PIECES], ids=["single", "drafts", "pieces"])
def test_attention(sizes, form, dtype):
    H, Hkv, d, page = form
    if sizes is PIECES and H > 8:
        sizes = [(1, 5), (131, 150), (40, 300), (0, 70)]
    Job(sizes, H=H, Hkv=Hkv, d=d, page=page, dtype=dtype, before=1, after=3, wider=2).check()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (17, 0), (100, 16), (128, 128), (129, 1), (200, 130), (1000, 4), (64, 1000)])
@pytest.mark.parametrize("sizes", [SINGLE, DRAFTS, PIECES], ids=["single", "drafts", "pieces"])
def test_attention_with_a_window_and_the_first_tokens(sizes, window, sinks, dtype):
    Job(sizes, H=4, Hkv=2, d=64, page=16, dtype=dtype, after=1).check(window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes", [SINGLE, PIECES], ids=["single", "pieces"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 3)])
def test_large_scores(sizes, window, sinks, dtype):
    """Scores of hundreds: rows whose weights all lie on one key, and a running maximum that grows along the way."""
    Job(sizes, H=2, Hkv=1, d=128, page=32, dtype=dtype, normal=30.0).check(window=window, sinks=sinks, scale=0.2)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("new", [1, 70])
def test_a_long_sequence(new, dtype):
    """Many keys for few rows: the work on one sequence is split over the keys."""
    Job([(new, 5000)], H=2, Hkv=1, d=64, page=64, dtype=dtype).check()
    Job([(new, 5000)], H=2, Hkv=1, d=64, page=64, dtype=dtype).check(window=3001, sinks=5)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("wider", [0, 4000], ids=["narrow", "wide"])  # which kernel has 17 to 64 rows goes by what the table can hold
@pytest.mark.parametrize("sizes", [
    [(4, 700), (1, 900), (0, 300), (2, 2), (16, 1500), (9, 40), (0, 0)],
    [(16, 2100)],
    [(1, 2100)],
    [(5, 600), (40, 1700), (3, 1), (1, 1), (5, 5), (129, 400)],
], ids=["drafts", "one", "one token", "mixed"])
@pytest.mark.parametrize("d,window,sinks", [(128, 0, 0), (64, 0, 0), (128, 300, 4)])
def test_between_few_and_many_rows(sizes, wider, d, window, sinks, dtype):
    sizes = [(min(n, length), length) for n, length in sizes]
    job = Job(sizes, H=32, Hkv=8, d=d, page=64, dtype=dtype, before=1, after=2, wider=wider)
    job.check(window=window, sinks=sinks)
    # a bound that more sequences might reach: other kernels, the same results
    job.check(window=window, sinks=sinks, max_new=min(job.T, max(n for n, _ in sizes) + 3))


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes,form,window", [
    ([(300, 5000), (1, 700), (260, 2900)], (4, 4, 128), 0),
    ([(300, 5000), (0, 0), (129, 130), (1, 1), (257, 2500)], (6, 2, 64), 0),
    ([(515, 4000), (200, 4100)], (8, 2, 128), 1900),
    ([(1030, 3000)], (40, 10, 64), 0),
])
def test_batches_in_pieces(sizes, form, window, dtype):
    H, Hkv, d = form
    Job(sizes, H=H, Hkv=Hkv, d=d, page=32, dtype=dtype, after=1).check(window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("form", [(71, 1, 64, 16), (96, 1, 128, 32), (22, 2, 64, 64)])
def test_many_query_heads_of_a_kv_head(form, dtype):
    H, Hkv, d, page = form
    Job([(1, 200), (2, 5), (0, 3), (3, 131)], H=H, Hkv=Hkv, d=d, page=page, dtype=dtype, after=2).check()
    Job([(1, 150)], H=H, Hkv=Hkv, d=d, page=page, dtype=dtype).check(max_new=1)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_more_sequences_than_are_put_in_order(dtype):
    sizes = [(n, n + 3 * b) for b, n in enumerate([40, 1, 0, 33, 70, 2, 65] * 10)]
    Job(sizes, H=2, Hkv=1, d=64, dtype=dtype, before=3, after=1).check()
    Job(sizes, H=2, Hkv=1, d=64, dtype=dtype).check(window=50, sinks=2)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes", [SINGLE, PIECES], ids=["single", "pieces"])
def test_tokens_of_very_different_size(sizes, dtype):
    """Keys and values whose rows differ by factors of up to 2^20: in 8 bits they have different powers of two."""
    job = Job(sizes, H=4, Hkv=2, d=64, dtype=dtype)
    g = torch.Generator().manual_seed(7)
    for x in (job.all_k, job.all_v):
        x.mul_(torch.exp2(torch.randint(-10, 11, (x.shape[0], x.shape[1], 1), generator=g).float()).cuda().to(BF16))
    s2a.s2a_cache_write(job.cache, job.all_k, job.all_v, job.table, job.all_starts, job.lengths)
    job.q *= 2.0**-6
    job.check()
    job.check(window=100, sinks=20)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("new", [40, 130])
def test_split_pieces_join_to_the_same_result(new, dtype):
    """One sequence whose items are split over their keys if there is a workspace, whatever that holds."""
    job = Job([(new, 3333)], H=4, Hkv=2, d=128, page=32, dtype=dtype, after=1)
    rows = job.rows().cuda()
    cache, batch = _structs(job)
    need = s2a.load().s2a_paged_workspace_bytes(cache, batch, 4, new, 0, 0)
    assert need > 0
    job.check()
    want = [t.clone() for t in job.attend()]
    for bytes_, bits in ((need, True), (need + 1000, True), (need - 1, False), (0, False)):
        ws = torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda")
        job.check(workspace=ws)
        got = job.attend(workspace=ws)
        assert not bits or (torch.equal(got[0][rows], want[0][rows]) and torch.equal(got[1][:, rows], want[1][:, rows]))


def _structs(job):
    """The two structs of include/s2a.h, as a program that calls the library through ctypes fills them in."""
    import ctypes

    class Cache(ctypes.Structure):
        _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_exp", "v_exp")] + [(n, ctypes.c_int) for n in ("type", "pages", "Hkv", "page_size", "d")]

    class Batch(ctypes.Structure):
        _fields_ = [(n, ctypes.c_void_p) for n in ("table", "starts", "lengths")] + [(n, ctypes.c_int) for n in ("width", "B", "T")]

    c, e4m3 = job.cache, job.dtype == E4M3
    cache = Cache(c.k.data_ptr(), c.v.data_ptr(), c.k_exp.data_ptr() if e4m3 else None, c.v_exp.data_ptr() if e4m3 else None, int(e4m3), *c.k.shape)
    batch = Batch(*(t.data_ptr() for t in job.where), job.table.shape[1], len(job.sizes), job.T)
    return ctypes.byref(cache), ctypes.byref(batch)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_the_library_is_called_directly(dtype):
    for sizes in (SINGLE, PIECES):
        job = Job(sizes, H=4, Hkv=2, d=64, dtype=dtype)
        want = job.attend()
        cache, batch = _structs(job)
        got = torch.full_like(want[0], 7), torch.full_like(want[1], 7)
        rc = s2a.load().s2a_paged_fwd(job.q.data_ptr(), cache, batch, got[0].data_ptr(), got[1].data_ptr(), 4, max(n for n, _ in sizes), 0.125, 0, 0, None, 0,
                                      torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_pages_beyond_two_to_the_31_values(dtype):
    """A pool of more than 2^32 values whose last pages are used: offsets pass 32 bits, row numbers do not."""
    H, Hkv, d, page = 4, 2, 128, 128
    small = Job([(1, 300), (150, 290), (2, 140)], H=H, Hkv=Hkv, d=d, page=page, dtype=dtype)
    pages = (1 << 32) // (Hkv * page * d) + 40
    big = s2a.PagedCache.empty(pages, Hkv, page, d, dtype)
    assert big.k.numel() > 1 << 32
    table = torch.arange(pages - 1, pages - 1 - small.table.numel(), -1, dtype=torch.int32, device="cuda").view(small.table.shape)
    s2a.s2a_cache_write(big, small.all_k, small.all_v, table, small.all_starts, small.lengths)
    for x in ("k", "v"):  # what the last pages hold past the ends
        getattr(big, x)[pages - 1 - table.numel()].view(torch.uint8).fill_(255)
    k, v = s2a.s2a_cache_read(big, table, small.all_starts, small.lengths, tokens=small.all_k.shape[0])
    wk, wv = s2a.s2a_cache_read(small.cache, small.table, small.all_starts, small.lengths, tokens=small.all_k.shape[0])
    assert torch.equal(k, wk) and torch.equal(v, wv)
    want = small.attend()
    got = s2a.s2a_paged_fwd(small.q, big, table, small.starts, small.lengths, max_new=150)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and s2a.device_status() == (0, 0)


def test_a_nan_stays_in_its_sequence():
    for sizes, dtype in ((SINGLE, BF16), (PIECES, BF16), (SINGLE, E4M3), (PIECES, E4M3)):
        job = Job(sizes, H=4, Hkv=2, d=64, dtype=dtype)
        want = [t.clone() for t in job.attend()]
        b = len(sizes) - 2 if sizes[-1][0] == 0 else 1
        n, length = sizes[b]
        page, slot = int(job.table[b, (length - n) // job.page]), (length - n) % job.page
        for x in (job.cache.k, job.cache.v):
            x[page, :, slot].view(torch.uint8).fill_(255)
        got = job.attend()
        rows = torch.ones(job.T, dtype=torch.bool, device="cuda")
        rows[int(job.starts[b]):int(job.starts[b + 1])] = False
        assert torch.equal(got[0][rows], want[0][rows]) and torch.equal(got[1][:, rows], want[1][:, rows])
        assert torch.isnan(got[0][~rows].float()).any()


def test_a_loose_bound_on_the_new_tokens_changes_no_more_than_roundings():
    for sizes in (SINGLE, DRAFTS):
        job = Job(sizes, H=4, Hkv=2, d=128)
        job.check(max_new=job.T)
        job.check(max_new=min(20, job.T))


def test_the_same_call_gives_the_same_bits():
    for sizes, dtype in ((SINGLE, BF16), (DRAFTS, E4M3), (PIECES, BF16), (PIECES, E4M3)):
        job = Job(sizes, H=8, Hkv=2, d=128, dtype=dtype)
        first = [t.clone() for t in job.attend()]
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, job.attend()))


def test_sequences_may_share_pages():
    job = Job([(1, 200), (1, 200), (1, 130)], H=4, Hkv=4, d=64, page=64)
    job.table[1] = job.table[0]
    job.table[2, :2] = job.table[0, :2]
    job.check()


# ---------------------------------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_a_prompt_in_pieces_and_then_single_tokens(dtype):
    """Two prompts go into the cache in pieces and are continued token by token; the result is that of the causal attention of the whole
    sequences (s2a_fwd_ex with one group), on the values that the cache stands for."""
    H, Hkv, d, page, N = 8, 2, 64, 16, 384
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(2, N, h, d, generator=g).to(BF16).cuda() for h in (H, Hkv, Hkv))
    cache = s2a.PagedCache.empty(2 * N // page, Hkv, page, d, dtype)
    table = torch.randperm(2 * N // page, generator=g).to(torch.int32).view(2, -1).cuda()
    o = torch.empty_like(q)
    lse = torch.empty((2, H, N), device="cuda")
    done = [0, 0]
    for step in [(200, 1), (129, 255), (0, 100)] + [(1, 1)] * 28 + [(27, 0)]:
        rows = [slice(done[b], done[b] + step[b]) for b in range(2)]
        starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, step[0], sum(step)], [done[b] + step[b] for b in range(2)]))
        new = [torch.cat([x[b, rows[b]] for b in range(2)]) for x in (q, k, v)]
        s2a.s2a_cache_write(cache, new[1], new[2], table, starts, lengths)
        got, got_lse = s2a.s2a_paged_fwd(new[0], cache, table, starts, lengths, max_new=max(step))
        for b, at in enumerate((slice(0, step[0]), slice(step[0], sum(step)))):
            o[b, rows[b]], lse[b, :, rows[b]] = got[at], got_lse[:, at]
            done[b] += step[b]
    assert done == [N, N]
    all_starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, N, 2 * N], [N, N]))
    held = [x.view(2, N, Hkv, d) for x in s2a.s2a_cache_read(cache, table, all_starts, lengths, tokens=2 * N)]
    if dtype == BF16:
        assert torch.equal(held[0], k) and torch.equal(held[1], v)
    want, want_lse = s2a.s2a_fwd_ex(q, *held, N, n_unshifted=H, shift=0)
    assert s2a.device_status() == (0, 0)
    # two results that each have rounded weights and themselves to bf16: 4 * 2^-8 of sum w |v|, which is at most max |v|
    assert float((o.float() - want.float()).abs().max()) <= 4 * 2.0**-8 * float(held[1].float().abs().max())
    assert float((lse - want_lse).abs().max()) <= 2e-4


def test_a_captured_step_follows_the_lengths():
    """A decoding loop as one captured step: starts, lengths and the table are read when the graph runs."""
    job = Job([(1, 100), (1, 30), (1, 1)], H=4, Hkv=2, d=128, wider=2)
    most = job.table.shape[1] * job.page
    for b in range(3):  # pages for every position of the table
        job.table[b] = torch.arange(job.table.shape[1], dtype=torch.int32) + b * job.table.shape[1]
    job.cache = s2a.PagedCache.empty(3 * job.table.shape[1], 2, 16, 128)
    job.cache.k.normal_(), job.cache.v.normal_()
    new_k, new_v = (torch.randn(3, 2, 128, device="cuda").to(BF16) for _ in range(2))

    def step():
        s2a.s2a_cache_write(job.cache, new_k, new_v, *job.where)
        return s2a.s2a_paged_fwd(job.q, job.cache, *job.where, max_new=1)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for lengths in ([100, 30, 1], [101, 31, 2], [most, 1, 57]):
        job.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        job.q.normal_(), new_k.normal_(), new_v.normal_()
        graph.replay()
        replayed = [t.clone() for t in got]
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(replayed, want))
    assert s2a.device_status() == (0, 0)


def test_a_captured_step_of_pieces_and_single_tokens():
    """A server's step captured once, with room for 40 new tokens of each sequence; starts and lengths change between the replays."""
    for B in (1, 3):
        job = Job([(40, 2000)] * B, H=4, Hkv=2, d=64, dtype=E4M3)
        T = job.T
        k, v = (torch.randn(T, 2, 64, device="cuda").to(BF16) for _ in range(2))
        o = torch.zeros_like(job.q)

        def step():
            s2a.s2a_cache_write(job.cache, k, v, *job.where)
            return s2a.s2a_paged_fwd(job.q, job.cache, *job.where, max_new=40, o=o)

        step()
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                got = step()
        for new in ([40] * B, [1] * B, [0] * (B - 1) + [39]):
            job.starts.copy_(torch.tensor([0] + [sum(new[:b + 1]) for b in range(B)], dtype=torch.int32))
            job.lengths.copy_(torch.tensor([1500 + n for n in new], dtype=torch.int32))
            job.q.normal_(), k.normal_(), v.normal_()
            graphs[0].replay()
            graphs[1].replay()
            replayed, rows = got[0].clone(), sum(new)
            want = step()
            assert torch.equal(replayed[:rows], want[0][:rows])
    assert s2a.device_status() == (0, 0)


def test_calls_from_several_threads():
    import threading

    jobs = [(Job(sizes, H=4, Hkv=2, d=64, dtype=dtype, seed=seed), torch.cuda.Stream()) for seed, (sizes, dtype) in
            enumerate([(SINGLE, BF16), (PIECES, E4M3), ([(130, 3000)], BF16), (DRAFTS, E4M3)])]
    want = [[t.clone() for t in job.attend()] for job, _ in jobs]
    torch.cuda.synchronize()
    failed = []

    def work(job, stream, want):
        try:
            rows = job.rows().cuda()
            for _ in range(20):
                o, lse = job.attend(stream=stream)
                stream.synchronize()
                failed.extend([1] if not (torch.equal(o[rows], want[0][rows]) and torch.equal(lse[:, rows], want[1][:, rows])) else [])
        except Exception as e:  # noqa: BLE001 - reported below
            failed.append(e)

    threads = [threading.Thread(target=work, args=(job, stream, w)) for (job, stream), w in zip(jobs, want)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not failed and s2a.device_status() == (0, 0)


def test_an_expired_wait_stops_the_paged_calls_too():
    job = Job(SINGLE, H=4, Hkv=2, d=64)
    o = torch.full((job.T, 4, 64), 7.0, dtype=BF16, device="cuda")
    s2a.selftest_wait_expiry(20_000_000)
    job.attend(o=o)
    torch.cuda.synchronize()
    assert (o == 7).all()
    with pytest.raises(s2a.S2AError) as e:
        job.attend()
    assert e.value.status == s2a.S2A_ERR_TIMEOUT and s2a.device_status()[0] == s2a.S2A_ERR_TIMEOUT
    job.check()


def test_another_stream():
    for sizes in (SINGLE, PIECES):
        job = Job(sizes, H=4, Hkv=2, d=64)
        want = [t.clone() for t in job.attend()]
        rows = job.rows().cuda()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)
        got = job.attend(stream=side)
        side.synchronize()
        assert torch.equal(got[0][rows], want[0][rows]) and torch.equal(got[1][:, rows], want[1][:, rows])


def test_results_have_the_class_of_q():
    class Marked(torch.Tensor):
        pass

    job = Job([(1, 20)])
    o, lse = s2a.s2a_paged_fwd(job.q.as_subclass(Marked), job.cache, *job.where)
    assert type(o) is Marked and type(lse) is torch.Tensor
    assert type(s2a.s2a_cache_read(job.cache, *job.where, tokens=1)[0]) is torch.Tensor


def test_refusals_reach_the_caller():
    job = Job([(2, 20)], H=4, Hkv=2)
    for kw in (dict(max_new=3), dict(max_new=0), dict(scale=-1.0), dict(window=-1), dict(sinks=1 << 40)):
        with pytest.raises(s2a.S2AError) as e:
            job.attend(**kw)
        assert e.value.status == s2a.S2A_ERR_INVALID_ARG
    with pytest.raises(s2a.S2AError) as e:
        s2a.s2a_paged_fwd(job.q[:, :3].contiguous(), job.cache, *job.where)  # 3 heads on 2
    assert e.value.status == s2a.S2A_ERR_INVALID_ARG
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        s2a.s2a_paged_fwd(job.q.cpu(), job.cache, *job.where)
    with pytest.raises(ValueError, match="lse must have dtype"):
        job.attend(lse=torch.empty((4, 2), dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError, match="workspace must have dtype"):
        job.attend(workspace=torch.empty(100, device="cuda"))
    with pytest.raises(s2a.S2AError) as e:
        job.attend(workspace=torch.empty(1024, dtype=torch.uint8, device="cuda")[16:])
    assert e.value.status == s2a.S2A_ERR_INVALID_ARG
    with pytest.raises(ValueError, match="tokens must be"):
        s2a.s2a_cache_read(job.cache, *job.where, tokens=-1)
    cache = s2a.PagedCache.empty(2, 2, 24, 64)
    with pytest.raises(s2a.S2AError) as e:
        s2a.s2a_paged_fwd(job.q, cache, *job.where)
    assert e.value.status == s2a.S2A_ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes", [[(1, 40), (1, 100)], [(1, 40), (150, 190)], [(40, 3000), (36, 2500)]], ids=["single", "pieces", "split pieces"])
@pytest.mark.parametrize("what", ["page", "negative page", "length", "short length", "starts", "new"])
def test_values_out_of_range_are_reported_and_not_followed(what, sizes, dtype):
    job = Job(sizes, H=4, Hkv=2, d=64, dtype=dtype)
    kw, code = {}, {"page": 1003, "negative page": 1003, "length": 1002, "short length": 1002, "starts": 1001, "new": 1004}[what]
    n = sizes[1][0]
    if what == "page":
        job.table[1, 1] = job.cache.k.shape[0]
    elif what == "negative page":
        job.table[1, 1] = -1
    elif what == "length":
        job.lengths[1] = job.table.shape[1] * job.page + 1
    elif what == "short length":
        job.lengths[1] = n - 1
    elif what == "starts":
        job.starts[1] = job.T + 1
    else:
        job.starts.copy_(torch.tensor([0, 0, n + 1], dtype=torch.int32))
        kw = dict(max_new=n)
    job.attend(**kw)
    torch.cuda.synchronize()
    with pytest.raises(s2a.S2AError) as e:  # nothing more until it has been read
        job.attend()
    assert e.value.status == s2a.S2A_ERR_BAD_INDEX
    assert s2a.device_status() == (s2a.S2A_ERR_BAD_INDEX, code) and s2a.device_status() == (0, 0)
    if what != "new":
        bad_read = dict(k=torch.zeros(job.T, 2, 64, dtype=BF16, device="cuda"), v=torch.zeros(job.T, 2, 64, dtype=BF16, device="cuda"))
        s2a.s2a_cache_read(job.cache, *job.where, **bad_read)
        # the bad page holds none of the new tokens
        assert s2a.device_status() == ((0, 0) if "page" in what else (s2a.S2A_ERR_BAD_INDEX, code))
