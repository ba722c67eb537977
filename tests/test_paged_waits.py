"""The paged cache's kernels keep the rules of tests/test_waits.py: lanes wait alone only where one lane runs, and no wait that can give up
stands between a store to tensor memory and the wait for it."""
import os
import re

import pytest
import test_waits


@pytest.mark.parametrize("name", ["paged_fwd.cu", "paged_split.cu"])
def test_lanes_wait_alone_only_where_one_lane_runs(name):
    test_waits.test_lanes_wait_alone_only_where_one_lane_runs(name)


@pytest.mark.parametrize("codes", [False, True])
def test_no_wait_can_give_up_on_stores_to_tensor_memory(codes):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(test_waits.CSRC, "paged_fwd.cu")).read())
    text = text.replace("if constexpr (!kE4M3)", "if constexpr (not kE4M3)")
    text = test_waits._inlined(test_waits._instance(text, dict(kE4M3=codes, kHalf=False, kWrite=False)))
    stores, pending = 0, 0
    for m in re.finditer(r"\btmem_st_\w+\(|\btmem_wait_st\(|\b(?:mbar_wait\w*|next_item)\(|\bnamed_barrier\w*\(", text):
        token = m.group()
        if token.startswith("tmem_st_"):
            stores, pending = stores + 1, pending + 1
        elif token.startswith("tmem_wait_st"):
            pending = 0
        else:
            assert pending == 0, f"{token} after stores to tensor memory that are not waited for"
    assert stores > 0 and pending == 0
