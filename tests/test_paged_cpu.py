"""The paged cache without a GPU: its index arithmetic (host-only C++), the oracle's own pins, and what the binding and the library
refuse before anything is enqueued."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

from oracle import paged_torch as ref
from paper_2309_12307_b200 import binding as s2a

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2309_12307_b200", "csrc")
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(CUDA_INC), reason="needs g++ and the CUDA headers")
def test_index_arithmetic(tmp_path):
    exe = str(tmp_path / "paged_index")
    src = os.path.join(ROOT, "tests", "host", "paged_index.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-I", CUDA_INC, src, "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


# ---------------------------------------------------------------------------------------------- the oracle
def test_oracle_code_values_are_those_of_torch():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(ref.code_values(), nan=1e9), torch.nan_to_num(want, nan=1e9))


def test_oracle_quantises_to_the_nearest_code():
    g = torch.Generator().manual_seed(1)
    for scale in (1.0, 2.0**-130, 2.0**100, 1e-3):
        row = (torch.randn(64, generator=g) * scale).to(torch.bfloat16)
        codes, e = ref.quantised_row(row)
        back = ref.code_values()[codes.long()] * math.ldexp(1.0, e)
        every = ref.code_values()[:127] * math.ldexp(1.0, e)
        every = torch.cat((every, -every))
        nearest = (row.double()[:, None] - every).abs().amin(1)
        assert torch.equal((row.double() - back).abs(), nearest)
        # half a step of the value, or of the smallest normal one
        assert ((row.double() - back).abs() <= torch.maximum(row.double().abs() * 2.0**-4, torch.tensor(math.ldexp(1.0, e - 10)))).all()
    assert ref.quantised_row(torch.zeros(64))[1] == -126
    assert ref.quantised_row(torch.tensor([1.0, math.inf]))[1] == ref.NOT_FINITE


def test_oracle_attends_like_one_softmax_over_the_whole_sequence():
    g = torch.Generator().manual_seed(2)
    L, n, H, Hkv, d, page = 37, 5, 4, 2, 8, 16
    k, v, q = (torch.randn(L, h, d, generator=g, dtype=torch.float64) for h in (Hkv, Hkv, H))
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
    cache = {x: torch.full((4, Hkv, page, d), math.nan, dtype=torch.float64) for x in "kv"}
    for t in range(L):
        cache["k"][table[0, t // page], :, t % page] = k[t]
        cache["v"][table[0, t // page], :, t % page] = v[t]
    starts, lengths = [1, 1 + n], [L]
    for window, sinks in ((0, 0), (7, 0), (7, 3), (100, 5), (1, 0)):
        o, lse, size, _ = ref.paged_fwd(torch.cat((q[:1], q[-n:], q[:1])), cache, table, starts, lengths, 0.3, window, sinks)
        assert torch.isnan(o[0]).all() and torch.isnan(o[-1]).all() and torch.isnan(lse[:, 0]).all()
        i, j = torch.arange(L)[:, None], torch.arange(L)[None]
        mask = (j <= i) & ((i - j < window) | (j < sinks) if window else True)
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(2, 1)) * 0.3
        s = s.masked_fill(~mask, -math.inf)
        p = s.softmax(-1)
        want = torch.einsum("hij,jhd->ihd", p, v.repeat_interleave(2, 1))[-n:]
        assert torch.allclose(o[1:-1], want, atol=1e-12) and torch.allclose(lse[:, 1:-1], s.logsumexp(-1)[:, -n:], atol=1e-12)
        assert (size[1:-1] >= want.abs() - 1e-12).all()


# ---------------------------------------------------------------------------------------------- refusals
def _cpu(codes=False):
    cache = s2a.PagedCache.empty(4, 2, 16, 64, torch.float8_e4m3fn if codes else torch.bfloat16, device="cpu")
    table, starts, lengths = (torch.zeros(s, dtype=torch.int32) for s in ((3, 2), (4,), (3,)))
    return cache, torch.zeros((5, 2, 64), dtype=torch.bfloat16), (table, starts, lengths)


def test_cpu_tensors_are_refused_before_the_library_is_called():
    cache, k, where = _cpu()
    for call in (lambda: s2a.s2a_cache_write(cache, k, k, *where), lambda: s2a.s2a_cache_read(cache, *where, tokens=5),
                 lambda: s2a.s2a_paged_fwd(k, cache, *where)):
        with pytest.raises(ValueError, match="cache.k must be a CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="must be a PagedCache"):
        s2a.s2a_paged_fwd(k, (k, k), *where)
    with pytest.raises(ValueError, match="tokens is needed"):
        s2a.s2a_cache_read(cache, *where)
    with pytest.raises(ValueError, match="float8_e4m3fn, not"):
        s2a.PagedCache.empty(4, 2, 16, 64, torch.float16, device="cpu")


@pytest.mark.parametrize("codes", [False, True])
def test_the_argument_checker_names_each_tensor(codes, monkeypatch):
    """The checks themselves, on CPU tensors (that they must be CUDA tensors was shown above to come first)."""
    real = s2a._require
    monkeypatch.setattr(s2a, "_require", lambda t, dtype, name, shape=None, device=None, cuda=True: real(t, dtype, name, shape, device, cuda=False))
    cache, k, (table, starts, lengths) = _cpu(codes)
    q = torch.zeros((5, 6, 64), dtype=torch.bfloat16)

    def changed(**kw):
        c = s2a.PagedCache(cache.k, cache.v, cache.k_exp, cache.v_exp)
        for name, t in kw.items():
            setattr(c, name, t)
        return c

    s2a._check_paged_fwd(q, cache, table, starts, lengths, None, None)
    s2a._check_cache_write(cache, k, k, table, starts, lengths)
    s2a._check_cache_read(cache, table, starts, lengths, 5, k, None)
    bad = [("cache.v must have shape", changed(v=cache.v[:3])), ("cache.k must be", changed(k=cache.k[0])), ("cache.k must have dtype", changed(k=cache.k.half())),
           ("cache.v must be contiguous", changed(v=cache.v.transpose(0, 2).contiguous().transpose(0, 2)))]
    if codes:
        bad += [("cache.k_exp must be a torch.Tensor", changed(k_exp=None)), ("cache.v_exp must have dtype", changed(v_exp=cache.v_exp.int())),
                ("cache.v_exp must have shape", changed(v_exp=cache.v_exp[:2]))]
    else:
        bad += [("cache.k_exp belongs to", changed(k_exp=torch.zeros((4, 2, 16), dtype=torch.int8)))]
    for message, c in bad:
        with pytest.raises(ValueError, match=message):
            s2a._check_paged_fwd(q, c, table, starts, lengths, None, None)
    for message, args in [("table must have dtype", (table.long(), starts, lengths)), ("table must be", (table[0], starts, lengths)),
                          ("starts must have shape", (table, starts[:3], lengths)), ("lengths must have shape", (table, starts, starts)),
                          ("lengths must have dtype", (table, starts, lengths.long()))]:
        with pytest.raises(ValueError, match=message):
            s2a._check_paged_fwd(q, cache, *args, None, None)
    where = table, starts, lengths
    for message, call in [("q must be", lambda: s2a._check_paged_fwd(q[..., :32].contiguous(), cache, *where, None, None)),
                          ("q must have dtype", lambda: s2a._check_paged_fwd(q.float(), cache, *where, None, None)),
                          ("o must have shape", lambda: s2a._check_paged_fwd(q, cache, *where, q[:4], None)),
                          ("lse must have shape", lambda: s2a._check_paged_fwd(q, cache, *where, None, torch.zeros((5, 6)))),
                          ("k must be", lambda: s2a._check_cache_write(cache, q, q, *where)),
                          ("v must have shape", lambda: s2a._check_cache_write(cache, k, k[:4], *where)),
                          ("v must have shape", lambda: s2a._check_cache_read(cache, *where, 5, k, k[:4])),
                          ("tokens must be", lambda: s2a._check_cache_read(cache, *where, -1, None, None))]:
        with pytest.raises(ValueError, match=message):
            call()


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_exp", "v_exp")] + [(n, ctypes.c_int) for n in ("type", "pages", "Hkv", "page_size", "d")]


class Batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("table", "starts", "lengths")] + [(n, ctypes.c_int) for n in ("width", "B", "T")]


def test_the_library_refuses_without_a_device():
    from paper_2309_12307_b200 import build

    lib = ctypes.CDLL(build.build())
    P, I = ctypes.c_void_p, ctypes.c_int
    lib.s2a_paged_fwd.argtypes = [P, P, P, P, P, I, I, ctypes.c_float, I, I, P, ctypes.c_size_t, P]
    lib.s2a_cache_write.argtypes = lib.s2a_cache_read.argtypes = [P] * 5
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 255) & ~255  # never dereferenced on these paths

    def call(cache=(), batch=(), q=a, o=a, lse=a, H=4, max_new=1, scale=1.0, window=0, sinks=0, workspace=None):
        c = Cache(**{**dict(k=a, v=a, k_exp=a, v_exp=a, type=1, pages=4, Hkv=2, page_size=16, d=64), **dict(cache)})
        b = Batch(**{**dict(table=a, starts=a, lengths=a, width=2, B=3, T=5), **dict(batch)})
        attend = lib.s2a_paged_fwd(q, ctypes.byref(c), ctypes.byref(b), o, lse, H, max_new, scale, window, sinks, workspace, 0, None)
        return attend, lib.s2a_cache_write(q, o, ctypes.byref(c), ctypes.byref(b), None), lib.s2a_cache_read(ctypes.byref(c), ctypes.byref(b), q, o, None)

    invalid, unsupported = s2a.S2A_ERR_INVALID_ARG, s2a.S2A_ERR_UNSUPPORTED
    for change in (dict(k=None), dict(v=a + 2), dict(k_exp=None), dict(v_exp=a + 8), dict(type=2), dict(type=-1), dict(pages=0), dict(Hkv=0), dict(d=-64),
                   dict(page_size=0)):
        assert call(cache=change) == (invalid,) * 3, change
    for change in (dict(d=96), dict(page_size=8), dict(page_size=24), dict(page_size=512), dict(pages=1 << 27)):
        assert call(cache=change) == (unsupported,) * 3, change
    for change in (dict(table=None), dict(starts=None), dict(lengths=None), dict(B=0), dict(T=0), dict(width=-1)):
        assert call(batch=change) == (invalid,) * 3, change
    for change in (dict(T=1 << 29, B=1), dict(width=1 << 27)):
        assert call(batch=change) == (unsupported,) * 3, change
    for change in (dict(q=None), dict(o=a + 8)):
        assert call(**change) == (invalid,) * 3, change
    for change in (dict(lse=a + 4), dict(lse=None), dict(H=3), dict(H=0), dict(max_new=0), dict(max_new=6), dict(scale=0.0), dict(scale=float("nan")),
                   dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(workspace=a + 16)):
        assert call(**change)[0] == invalid, change
    assert lib.s2a_cache_write(a, a, None, None, None) == invalid and lib.s2a_paged_fwd(a, None, None, a, a, 4, 1, 1.0, 0, 0, None, 0, None) == invalid
