"""The paged cache without a GPU: host-only C++ checks of its masks and offsets."""
import os
import shutil
import subprocess

import pytest
from test_paged_cpu import CSRC, CUDA_INC, ROOT, _cpu

from paper_2309_12307_b200 import binding as s2a


def run_host(name, tmp_path):
    exe = str(tmp_path / name)
    src = os.path.join(ROOT, "tests", "host", name + ".cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-I", CUDA_INC, src, "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(CUDA_INC), reason="needs g++ and the CUDA headers")
@pytest.mark.parametrize("name", ["paged_hidden", "paged_table"])
def test_on_the_host(name, tmp_path):
    run_host(name, tmp_path)


@pytest.mark.parametrize("name", ["paged.h", "paged_fwd.cu", "paged_split.cu", "cache_kernels.cu"])
def test_entries_of_the_table_are_found_by_its_one_function(name):
    text = open(os.path.join(CSRC, name)).read()
    assert text.count("batch.table +") == text.count("batch.table + table_row(")


def _body(text, head):
    """The braces after `head`."""
    i = text.index("{", text.index(head))
    depth = 0
    for x in range(i, len(text)):
        depth += (text[x] == "{") - (text[x] == "}")
        if depth == 0:
            return text[i:x + 1]


def test_what_keeps_the_paged_kernels_from_running_keeps_no_other():
    """An error of the paged kernels' set-up is kept for s2a_paged_fwd; the device is ready all the same."""
    api, paged = (open(os.path.join(CSRC, name)).read() for name in ("api.cu", "api_paged.cu"))
    setup = _body(api, "int prepare_device(DeviceState** out)")
    for line in setup.splitlines():
        if "configure_paged" in line:
            assert "ds.paged_error = configure_paged" in line and "return" not in line
    assert setup.count("configure_paged") == 2 and "return cuda_fail(ds.paged_error)" not in setup and "cudaGetLastError();" in setup
    assert "prepare_paged(" in _body(paged, "int s2a_paged_fwd(") and "prepare_device(" not in _body(paged, "int s2a_paged_fwd(")
    assert "prepare_device(" in _body(paged, "int copy_impl(")


def test_no_rows_are_refused_with_the_range_that_the_library_takes(monkeypatch):
    real = s2a._require
    monkeypatch.setattr(s2a, "_require", lambda t, dtype, name, shape=None, device=None, cuda=True: real(t, dtype, name, shape, device, cuda=False))
    cache, _, where = _cpu()
    for tokens in (0, 1 << 31):
        with pytest.raises(ValueError, match=r"tokens must be in \[1, 2\^31\)"):
            s2a._check_cache_read(cache, *where, tokens, None, None)
    s2a._check_cache_read(cache, *where, 1, None, None)


def test_a_cache_of_a_derived_class_is_a_cache():
    class Marked(s2a.PagedCache):
        pass

    cache, k, where = _cpu(codes=True)
    marked = Marked(cache.k, cache.v, cache.k_exp, cache.v_exp)
    assert all(a is b for a, b in zip(s2a._pools(marked), (cache.k, cache.v, cache.k_exp, cache.v_exp)))
    assert s2a._pools((k, k)) == (None,) * 4
