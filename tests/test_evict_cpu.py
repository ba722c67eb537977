"""Weights of cached tokens and eviction without a GPU: the oracle's own pins, the order of weights, and what the library refuses before anything is enqueued."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch
from test_paged_cpu import CSRC, CUDA_INC, ROOT, Batch, Cache

from oracle import evict_torch as ref
from paper_2309_12307_b200 import binding as s2a


def test_oracle_weights_are_the_columns_of_the_softmax():
    g = torch.Generator().manual_seed(2)
    L, n, H, Hkv, d, page = 37, 5, 4, 2, 8, 16
    k, q = (torch.randn(L, h, d, generator=g, dtype=torch.float64) for h in (Hkv, H))
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
    cache = {"k": torch.full((4, Hkv, page, d), math.nan, dtype=torch.float64)}
    for t in range(L):
        cache["k"][table[0, t // page], :, t % page] = k[t]
    i, j = torch.arange(L - n, L)[:, None], torch.arange(L)[None]
    for window, sinks in ((0, 0), (7, 3)):
        mask = (j <= i) & ((i - j < window) | (j < sinks) if window else True)
        s = (torch.einsum("ihd,jhd->hij", q[-n:], k.repeat_interleave(2, 1)) * 0.3).masked_fill(~mask, -math.inf)
        want = s.softmax(-1).view(Hkv, 2, n, L).sum((1, 2))
        before = torch.rand(4, Hkv, page, generator=g)
        got, written = ref.paged_weights(q[-n:], s.logsumexp(-1), cache, table, [0, n], [L], torch.full((4, Hkv, page), -1.0), before, 0.3, window, sinks)
        for t in range(L):
            at = int(table[0, t // page]), slice(None), t % page
            seen = bool(mask[:, t].any())
            assert bool(written[at].all()) == seen
            assert torch.allclose(got[at], (want[:, t] + (before[at].double() if t < L - n else 0)) if seen else torch.tensor(-1.0, dtype=torch.float64))


def test_oracle_keeps_by_weight_then_by_place():
    assert ref.kept_tokens([1, 5, 5, 2, 5, 9], 3, 0, 0) == [1, 2, 5]
    assert ref.kept_tokens([1, 5, 5, 2, 5, 9], 3, 1, 1) == [0, 1, 5]
    assert ref.kept_tokens([1.0, math.nan, 5.0, 0.0, -0.0], 2, 0, 0) == [1, 2]
    assert ref.kept_tokens([0.0, -0.0, 0.0, -0.0], 2, 0, 0) == [0, 1]
    assert ref.kept_tokens([3, 2], 5, 1, 1) == [0, 1]


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(CUDA_INC), reason="needs g++ and the CUDA headers")
def test_order_of_weights(tmp_path):
    exe = str(tmp_path / "weight_order")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-I", CUDA_INC, os.path.join(ROOT, "tests", "host", "weight_order.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(CUDA_INC), reason="needs g++ and the CUDA headers")
def test_items_have_each_row_and_key_once(tmp_path):
    exe = str(tmp_path / "weight_items")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, "-I", CUDA_INC, os.path.join(ROOT, "tests", "host", "weight_items.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_cpu_tensors_are_refused_before_the_library_is_called():
    cache = s2a.PagedCache.empty(4, 2, 16, 64, device="cpu")
    table, starts, lengths = (torch.zeros(s, dtype=torch.int32) for s in ((3, 2), (4,), (3,)))
    received = torch.zeros(4, 2, 16)
    q = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: s2a.s2a_paged_weights(q, received, cache, table, starts, lengths, received), lambda: s2a.s2a_cache_evict(cache, received, table, lengths, table, 5)):
        with pytest.raises(ValueError, match="cache.k must be a CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="must be a PagedCache"):
        s2a.s2a_cache_evict(None, received, table, lengths, table, 5)


def test_the_library_refuses_without_a_device():
    lib = s2a.load()
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 255) & ~255  # never dereferenced on these paths

    def call(cache=(), batch=(), q=a, lse=a, received=a, before=None, H=4, max_new=1, scale=1.0, window=0, sinks=0, table=a, lengths=a, to_table=a, width=2, to_width=1, B=3, budget=16,
             recent=0, new_lengths=a + 256, kept=a, workspace=None):
        c = Cache(**{**dict(k=a, v=a, k_exp=a, v_exp=a, type=1, pages=4, Hkv=2, page_size=16, d=64), **dict(cache)})
        b = Batch(**{**dict(table=a, starts=a, lengths=a, width=2, B=3, T=5), **dict(batch)})
        return (lib.s2a_paged_weights(q, lse, ctypes.byref(c), ctypes.byref(b), before, received, H, max_new, scale, window, sinks, workspace, 0, None),
                lib.s2a_cache_evict(ctypes.byref(c), received, table, width, lengths, to_table, to_width, B, budget, sinks, recent, new_lengths, kept, None))

    invalid, unsupported = s2a.S2A_ERR_INVALID_ARG, s2a.S2A_ERR_UNSUPPORTED
    for change in (dict(k=None), dict(v=a + 2), dict(k_exp=None), dict(type=2), dict(pages=0), dict(Hkv=0), dict(page_size=0)):
        assert call(cache=change) == (invalid,) * 2, change
    for change in (dict(d=96), dict(page_size=24), dict(pages=1 << 27)):
        assert call(cache=change) == (unsupported,) * 2, change
    for change in (dict(table=None), dict(B=0), dict(T=0)):
        assert call(batch=change)[0] == invalid, change
    for change in (dict(received=None), dict(received=a + 4), dict(sinks=-1)):
        assert call(**change) == (invalid,) * 2, change
    for change in (dict(q=None), dict(q=a + 8), dict(lse=None), dict(lse=a + 4), dict(before=a + 4), dict(H=3), dict(max_new=0), dict(max_new=6), dict(scale=0.0), dict(scale=float("inf")),
                   dict(window=-1), dict(workspace=a + 16)):
        assert call(**change)[0] == invalid, change
    for change in (dict(table=None), dict(lengths=None), dict(to_table=None), dict(width=0), dict(to_width=0), dict(B=0), dict(budget=0), dict(recent=-1), dict(sinks=10, recent=7),
                   dict(sinks=2**31 - 1, recent=2**31 - 1), dict(budget=17), dict(new_lengths=None), dict(new_lengths=a), dict(new_lengths=a + 8), dict(kept=None)):
        assert call(**change)[1] == invalid, change
    for change in (dict(width=1 << 27, to_width=1 << 26), dict(to_width=1 << 27), dict(B=1 << 30, new_lengths=a + (1 << 40))):
        assert call(**change)[1] == unsupported, change
    assert call(budget=1 << 30, to_width=2)[1] == unsupported  # (places behind the last token are counted in an int)
    assert lib.s2a_paged_weights(a, a, None, None, None, a, 4, 1, 1.0, 0, 0, None, 0, None) == invalid
