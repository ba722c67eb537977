"""Attention over the paged cache on random batches, against its definition in 64 bits on the GPU: every head ratio, page size, window and mix of lengths
meets every other, and what must not matter is NaN or huge."""
import math
import random

import pytest
import torch
from test_gpu_paged import BF16, E4M3, Job, compare
from test_gpu_paged_edges import leave_behind

from oracle import paged_torch as ref
from paper_2309_12307_b200 import binding as s2a

pytestmark = pytest.mark.gpu


def sequence_values(job, x, b, length):
    """[Hkv, length, d] of sequence b, and the exponents of its rows (None in bf16)."""
    pages = job.table[b, :-(-length // job.page)].long()
    if job.dtype == BF16:
        values, e = getattr(job.cache, x)[pages].double(), None
    else:
        e = getattr(job.cache, x + "_exp")[pages].double()
        codes = getattr(job.cache, x).view(torch.uint8)[pages].long()
        values = ref.code_values().cuda()[codes] * torch.exp2(torch.where(e == ref.NOT_FINITE, math.nan, e))[..., None]
        e = e.transpose(0, 1).reshape(e.shape[1], -1)[:, :length]
    return values.transpose(0, 1).reshape(values.shape[1], -1, job.d)[:, :length], e


def reference(job, scale, window, sinks):
    """As oracle.paged_torch.paged_fwd."""
    T, H, d = job.q.shape
    o = torch.full((T, H, d), math.nan, dtype=torch.float64, device="cuda")
    size, lse = o.clone(), torch.full((H, T), math.nan, dtype=torch.float64, device="cuda")
    largest = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    starts = job.starts.tolist()
    for b, (n, length) in enumerate(job.sizes):
        if n == 0:
            continue
        rows, blocks = slice(starts[b], starts[b + 1]), -(-length // 128)
        (k, _), (v, e) = (sequence_values(job, x, b, length) for x in ("k", "v"))
        p, j = torch.arange(length - n, length, device="cuda")[:, None], torch.arange(length, device="cuda")[None]
        hidden = (j > p) | ((j <= p - window) & (j >= sinks) if window else j < 0)
        for h in range(H):
            hk = h // (H // k.shape[0])
            s = (scale * (job.q[rows, h].double() @ k[hk].T)).masked_fill(hidden, -math.inf)
            lse[h, rows] = torch.logsumexp(s, -1)
            w = torch.exp(s - lse[h, rows, None])
            o[rows, h], size[rows, h] = w @ v[hk], w @ v[hk].abs()
            if e is not None:
                powers, weights = (torch.zeros((x, blocks * 128), dtype=torch.float64, device="cuda") for x in (1, n))
                powers[0, :length], weights[:, :length] = torch.exp2(e[hk]), w
                largest[rows, h] = (weights.view(n, blocks, 128).amax(-1) * powers.view(1, blocks, 128).amax(-1)).amax(-1)
    return o.cpu(), lse.cpu(), size.cpu(), largest.cpu()


@pytest.mark.parametrize("seed", range(40))
def test_random_batches(seed):
    r = random.Random(seed)
    for _ in range(6):
        d, page, dtype = r.choice([64, 128]), r.choice([16, 32, 64, 128, 256]), r.choice([BF16, E4M3])
        Hkv = r.choice([1, 1, 2, 3, 5, 8])
        rep = min(80 // Hkv, r.choice([1, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 24, 71]))
        B, most = r.choice([1, 1, 2, 3, 6, 20, 70]), r.choice([1, 1, 4, 9, 40, 130, 300])
        longest, most = int(2 ** r.uniform(0, 12 if B < 5 else 9)), min(most, 40) if B >= 20 else most
        lengths = [r.randint(0, longest) for _ in range(B)]
        sizes = [(r.randint(0, min(length, most)), length) for length in lengths]
        if not any(n for n, _ in sizes):
            sizes[0] = 1, max(1, lengths[0])
        window, sinks = r.choice([0, 0, 1, r.randint(1, 300), r.randint(1, longest + 5)]), r.choice([0, 1, 4, r.randint(0, 300)])
        job = Job(sizes, H=Hkv * rep, Hkv=Hkv, d=d, page=page, dtype=dtype, before=r.choice([0, 0, 3]), after=r.choice([0, 0, 1, 5]), seed=r.randint(0, 1 << 30),
                  wider=r.choice([0, 0, 3, 1000]), normal=r.choice([1.0, 1.0, 8.0]))
        scale = r.choice([d**-0.5, 0.02])
        want = reference(job, scale, window, sinks)
        if window:
            leave_behind(job, window, sinks, r.choice(["nan", "large"]))
        kw = dict(max_new=min(job.T, max(n for n, _ in sizes) + r.choice([0, 0, 2, 100])))
        if r.random() < 0.3:
            kw["workspace"] = torch.empty(0, dtype=torch.uint8, device="cuda")
        o, lse = job.attend(scale=scale, window=window, sinks=sinks, o=torch.full((job.T, job.H, d), 7.0, dtype=BF16, device="cuda"),
                            lse=torch.full((job.H, job.T), 7.0, device="cuda"), **kw)
        assert s2a.device_status() == (0, 0)
        inside = job.rows()
        compare(o.cpu(), lse.cpu(), *want, inside, max(lengths), d, scale, float(job.q.cpu()[inside].double().norm(dim=-1).max()), job.all_k)
