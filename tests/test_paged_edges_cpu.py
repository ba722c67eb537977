"""The paged cache without a GPU: host-only C++ checks of its masks and offsets."""
import os
import shutil
import subprocess

import pytest
from test_paged_cpu import CSRC, CUDA_INC, ROOT


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
