"""The paged cache on the GPU at the edges of its number ranges and masks, against its definition in 64 bits."""
import math

import pytest
import torch
from test_gpu_paged import BF16, E4M3, PIECES, Job, compare

from oracle import paged_torch as ref
from paper_2309_12307_b200 import binding as s2a

pytestmark = pytest.mark.gpu


def refill(job):
    """all_k and all_v, as they are now, into the cache."""
    s2a.s2a_cache_write(job.cache, job.all_k, job.all_v, job.table, job.all_starts, job.lengths)


def zero_keys(job, which):
    """Keys of zeros: those of the whole sequences, of the last (ragged, masked) block of 128, or of the blocks with an odd number."""
    at = 0
    for _, length in job.sizes:
        j = torch.arange(length, device="cuda")
        last = j // 128 == max(0, length - 1) // 128
        job.all_k[at:at + length][{"all": j >= 0, "last": last, "odd": j // 128 % 2 == 1}[which]] = 0
        at += length
    refill(job)


# ---------------------------------------------------------------------------------------------- keys that are zero or tiny
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (129, 130)])
@pytest.mark.parametrize("which", ["all", "last", "odd"])
@pytest.mark.parametrize("d,scale", [(64, 64**-0.5), (128, 128**-0.5), (64, 1 / 64), (128, 2.0**-130)])
def test_blocks_of_keys_that_are_zero(d, scale, which, window, sinks, dtype):
    """Scores of zero beside masked ones, with small queries: what scores are multiplied with must not vanish."""
    for sizes, down in ((PIECES, 2.0**-10), ([(200, 3000)], 2.0**-2), ([(1, 1), (1, 129), (1, 300)], 2.0**-10)):
        job = Job(sizes, H=4, Hkv=2, d=d, page=16, dtype=dtype)
        zero_keys(job, which)
        job.q *= down
        job.check(scale=scale, window=window, sinks=sinks)


@pytest.mark.parametrize("new", [1, 30, 200])
@pytest.mark.parametrize("q_power,k_power", [(-100, 100), (100, -117), (120, -126), (-118, 118), (0, -120), (-120, 0)])
def test_queries_and_keys_at_the_ends_of_the_range(q_power, k_power, new):
    """8-bit keys whose powers of two and those of the queries cancel, or leave next to nothing."""
    for window, sinks in ((0, 0), (70, 3)):
        job = Job([(new, 300)], H=4, Hkv=2, d=64, page=32, dtype=E4M3)
        job.all_k *= 2.0**k_power
        refill(job)
        job.q *= 2.0**q_power
        job.check(window=window, sinks=sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 30, 200])
def test_scores_that_are_zero_between_the_largest_numbers(d, new):
    """Queries and keys near 2^127 with nothing in common: the scores are zero, whatever power of two they would be multiplied with."""
    job = Job([(new, 300)], H=4, Hkv=2, d=d, page=32, dtype=E4M3)
    job.all_k[..., :d // 2] = 0
    job.all_k[..., d // 2:] = 2.0**127
    job.q[..., d // 2:] = 0
    job.q[..., :d // 2] = 2.0**127
    refill(job)
    o, lse = job.attend(o=torch.full((job.T, 4, d), 7.0, dtype=BF16, device="cuda"), lse=torch.full((4, job.T), 7.0, device="cuda"))
    want = ref.paged_fwd(job.q.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), d**-0.5)
    # (no score is off: they are sums of zeros)
    compare(o.cpu(), lse.cpu(), *want, job.rows(), 300, d, d**-0.5, 0.0, torch.zeros(1))


def test_keys_marked_as_not_finite_reach_no_token_before_them():
    """The last block's keys are NaN throughout; tokens that attend none of them have what they have without it."""
    for d in (64, 128):
        job = Job([(150, 170)], H=4, Hkv=2, d=d, page=16, dtype=E4M3)
        job.q *= 2.0**-6
        want = [t.clone() for t in job.attend()]
        job.all_k[128:] = math.inf
        refill(job)
        o, lse = job.attend()
        # (new token i is at position 20 + i)
        assert torch.equal(o[:108], want[0][:108]) and torch.equal(lse[:, :108], want[1][:, :108])
        assert torch.isnan(lse[:, 108:]).all() and s2a.device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("scale", [2.0**-149, 2.0**-130, 2.0**-126, 2.0**127, 3e38])
def test_the_least_and_the_largest_scales(scale, dtype):
    for sizes, window in (([(1, 300), (30, 130)], 0), ([(200, 300)], 0), ([(200, 300), (1, 200)], 150)):
        job = Job(sizes, H=4, Hkv=2, d=64, page=16, dtype=dtype)
        if scale > 1:
            zero_keys(job, "all")
        job.check(scale=scale, window=window)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("power", [-100, -108, -115, -120, -126])
@pytest.mark.parametrize("sizes", [[(1, 300), (3, 40)], [(200, 300)], [(40, 3000)]], ids=["few", "pieces", "split pieces"])
def test_values_near_the_least_number(sizes, power, dtype):
    H, Hkv, d = 4, 2, 64
    job = Job(sizes, H=H, Hkv=Hkv, d=d, page=16, dtype=dtype)
    job.all_v *= 2.0**power
    refill(job)
    o, _ = job.attend()
    assert s2a.device_status() == (0, 0)
    want, _, size, largest = ref.paged_fwd(job.q.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), d**-0.5)
    score = d * 2.0**-24 * d**-0.5 * float(job.q.double().norm(dim=-1).max()) * float(job.all_k.double().norm(dim=-1).max()) + 2.0**-20
    longest = max(n for _, n in sizes)
    # as in compare(), without its absolute slack.  The result's step is 2^-133 and more; values of a tile are fp16 numbers, times 2^6 and 2^-e with e no
    # less than -100: steps of 2^-24 * 2^-106, half of one each (and as much again for sums in 32 bits that are as small).
    allowed = (2.0**-8 + 2 * score + longest * 2.0**-24) * size + 2.0**-8 * (want.abs() + 2.0**-8 * size) + 2.0**-134 + 2.0**-32 * 448 * longest * largest[..., None]
    allowed += 2.0**-130 if dtype == E4M3 else 2.0**-140
    off = (o.cpu().double() - want).abs()
    assert (off <= allowed).all(), float((off / allowed).max())


# ---------------------------------------------------------------------------------------------- rows stay by themselves
@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("sizes,power", [([(1, 300)], 20), ([(1, 300)], 40), ([(1, 300)], 100), ([(1, 40), (4, 500), (1, 1)], 20), ([(1, 40), (4, 500), (1, 1)], 40),
                                         ([(1, 40), (4, 500), (1, 1)], 100), ([(200, 500)], 20), ([(200, 500)], 40), ([(200, 500)], 100)])
def test_a_large_query_reaches_no_other_row(sizes, power, dtype):
    """One head's queries, and one token's, are 2^power times as large as the others of their KV head and sequence."""
    H, Hkv, d = 8, 2, 64
    job = Job(sizes, H=H, Hkv=Hkv, d=d, page=16, dtype=dtype)
    large = torch.zeros(job.T, H, dtype=torch.bool)
    large[:, 1] = True
    if job.T > 1:
        large[job.T // 2] = True
    job.q[large.cuda()] *= 2.0**power
    o, lse = job.attend()
    assert s2a.device_status() == (0, 0) and torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    want, want_lse, size, largest = ref.paged_fwd(job.q.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), d**-0.5)
    q_norm = float(job.q.cpu()[~large].double().norm(dim=-1).max())
    # the other rows, one after the other, as rows of one head
    flat = [x[~large][:, None] for x in (o.cpu(), want, size, largest)]
    rows = flat[0].shape[0]
    compare(flat[0], lse.cpu().T[~large][None], flat[1], want_lse.T[~large][None], flat[2], flat[3], torch.ones(rows, dtype=torch.bool), max(n for _, n in sizes), d, d**-0.5,
            q_norm, job.all_k)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("power", [0, 10, 14, 18, 22, 26, 30, 40, 90])
@pytest.mark.parametrize("sizes", [[(1, 300), (1, 1)], [(4, 300)], [(200, 500), (1, 40)]], ids=["one", "drafts", "pieces"])
def test_a_token_that_attends_itself_alone_has_its_own_value(sizes, power, dtype):
    """The weight of the only key is 1, however large its score: sums of weights and of weighted values must go by the same maximum."""
    H, Hkv, d = 4, 2, 64
    job = Job(sizes, H=H, Hkv=Hkv, d=d, page=16, dtype=dtype)
    job.q *= 2.0**power
    o, lse = job.attend(window=1)
    assert s2a.device_status() == (0, 0)
    _, held = s2a.s2a_cache_read(job.cache, *job.where, tokens=job.T)
    want = held.repeat_interleave(H // Hkv, 1).double()
    # the weight and the result are rounded, to 8 bits at least, half a step each; the exponential is off by 2^-20 and less
    assert ((o.double() - want).abs() <= (2 * 2.0**-8 + 2.0**-15) * want.abs()).all(), float(((o.double() - want).abs() / want.abs()).max())
    k, _ = s2a.s2a_cache_read(job.cache, *job.where, tokens=job.T)
    score = (job.q.double() * k.repeat_interleave(H // Hkv, 1).double()).sum(-1).T * d**-0.5
    most = (job.q.double().norm(dim=-1) * k.repeat_interleave(H // Hkv, 1).double().norm(dim=-1)).T * d**-0.5
    assert ((lse.double() - score).abs() <= most * d * 2.0**-24 + score.abs() * 2.0**-21 + 2.0**-20).all()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("power", [12, 20, 26, 30])
@pytest.mark.parametrize("sizes", [[(4, 100)], [(150, 170)], [(200, 3000)]], ids=["drafts", "pieces", "split pieces"])
def test_how_far_a_later_token_moves_earlier_ones(sizes, power, dtype):
    """The last token's k and v are 2^power times as large as the others'.  Only it attends itself; in 8 bits the tokens before it share its fp16 tile."""
    H, Hkv, d, page = 4, 2, 64, 16
    job = Job(sizes, H=H, Hkv=Hkv, d=d, page=page, dtype=dtype)
    length = sizes[0][1]
    others = job.all_k[:-1].clone()
    job.all_k[-1] *= 2.0**power
    job.all_v[-1] *= 2.0**power
    refill(job)
    o, lse = (t.cpu() for t in job.attend())
    assert s2a.device_status() == (0, 0)
    want, want_lse, size, largest = ref.paged_fwd(job.q.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), d**-0.5)
    inside = torch.ones(job.T, dtype=torch.bool)
    inside[-1] = False
    o[-1], lse[:, -1] = 7, 7

    def lost(exponents):
        """What a value of the last 128 rows is off by at most: a row goes to fp16 times 2^(e - most + 6), most the largest e.  An 8-bit float is a multiple of
        2^-9, so nothing is lost of multiples of 2^-24 (e >= most - 21).  Below that the product is rounded, by 2^-25 at most; and the factor, an
        fp16 number itself, is no less than 2^-24 or zero (e < most - 30: values up to 448 * 2^e go)."""
        j = torch.arange((length - 1) // 128 * 128, length)
        e = exponents.cpu()[job.table.cpu()[0, j // page].long(), :, j % page].double()
        off = torch.where(e >= e.max() - 21, 0.0, torch.where(e >= e.max() - 30, 2.0 ** (e.max() - 31), 448 * torch.exp2(e)))
        return float(off.max())

    off_k, off_v = (lost(job.cache.k_exp), lost(job.cache.v_exp)) if dtype == E4M3 and job.T > 16 else (0.0, 0.0)
    q_norm = float(job.q.double().norm(dim=-1).max())
    score = d**-0.5 * float(job.q.double().abs().sum(-1).max()) * off_k
    # compare() allows 2^-8 of `size`, and of scores what their sums in 32 bits are off by, d * 2^-24 * scale * |q| |k|
    size = size * (1 + 2.0**8 * 2 * score) + 2.0**8 * off_v
    k_norm = float(others.double().norm(dim=-1).max()) + score / (d * 2.0**-24 * d**-0.5 * q_norm)
    compare(o, lse, want, want_lse, size, largest, inside, length, d, d**-0.5, q_norm, torch.full((1, d), k_norm / math.sqrt(d), dtype=torch.float64))


# ---------------------------------------------------------------------------------------------- behind the window
def leave_behind(job, window, sinks, fill):
    """What no new token of a sequence attends, in front of its window, goes: table entries of whole pages, and the values of the other keys become
    NaN or the largest numbers there are (a page that was given back holds another sequence's tokens)."""
    table = job.table.cpu()
    for b, (n, length) in enumerate(job.sizes):
        low = max(0, length - n - window + 1)
        for i in range(-(-length // job.page)):
            gone = torch.tensor([sinks <= j < low for j in range(i * job.page, (i + 1) * job.page)]).cuda()
            page = int(table[b, i])
            if gone.all() and n > 0:
                table[b, i] = -1
            if n > 0:
                for x in ("k", "v"):
                    pool = getattr(job.cache, x)
                    pool[page][:, gone] = torch.tensor(math.nan if fill == "nan" else 3e38, device="cuda").to(pool.dtype) if job.dtype == BF16 else \
                        torch.full((), 127 if fill == "nan" else 126, dtype=torch.uint8, device="cuda").view(E4M3)
                    if job.dtype == E4M3:
                        getattr(job.cache, x + "_exp")[page][:, gone] = ref.NOT_FINITE if fill == "nan" else 119
    job.table.copy_(table)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("fill", ["nan", "large"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (33, 40), (100, 1), (129, 130)])
@pytest.mark.parametrize("form", [(4, 2, 64, 16), (4, 4, 128, 32), (8, 1, 64, 256)])
def test_what_lies_behind_a_window_does_not_matter(form, window, sinks, fill, dtype):
    H, Hkv, d, page = form
    for sizes in ([(1, 600), (1, 40), (4, 333)], [(150, 700), (1, 300), (0, 20), (70, 400)], [(40, 1500)]):
        job = Job(sizes, H=H, Hkv=Hkv, d=d, page=page, dtype=dtype, after=1)
        want, want_lse, size, largest = ref.paged_fwd(job.q.cpu(), job.host_cache(), job.table.cpu(), job.starts.cpu(), job.lengths.cpu(), d**-0.5, window, sinks)
        leave_behind(job, window, sinks, fill)
        o, lse = job.attend(window=window, sinks=sinks, o=torch.full((job.T, H, d), 7.0, dtype=BF16, device="cuda"), lse=torch.full((H, job.T), 7.0, device="cuda"))
        assert s2a.device_status() == (0, 0)
        compare(o.cpu(), lse.cpu(), want, want_lse, size, largest, job.rows(), max(n for _, n in sizes), d, d**-0.5, float(job.q.cpu()[job.rows()].double().norm(dim=-1).max()),
                job.all_k)


def test_no_rows_are_refused():
    job = Job([(1, 20)])
    with pytest.raises(ValueError, match="tokens must be in"):
        s2a.s2a_cache_read(job.cache, *job.where, tokens=0)
    empty = job.q[:0]
    for call in (lambda: s2a.s2a_paged_fwd(empty, job.cache, *job.where), lambda: s2a.s2a_cache_write(job.cache, empty[:, :2].contiguous(), empty[:, :2].contiguous(), *job.where)):
        with pytest.raises(s2a.S2AError) as e:
            call()
        assert e.value.status == s2a.S2A_ERR_INVALID_ARG


def test_a_cache_of_a_derived_class_is_a_cache():
    class Marked(s2a.PagedCache):
        pass

    job = Job([(1, 20), (3, 40)])
    want = [t.clone() for t in job.attend()]
    job.cache = Marked(job.cache.k, job.cache.v, job.cache.k_exp, job.cache.v_exp)
    assert all(torch.equal(a, b) for a, b in zip(want, job.attend()))
