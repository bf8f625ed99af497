"""Attention over pools in 8 bits and the selection of a beam search: a wave has waited for its chip-coherent stores where its workgroup counts itself in (as
test_arrivals.py checks it for the other kernels of that kind; no GPU needed)."""
import re

import pytest

from test_arrivals import arrivals, listing


@pytest.mark.parametrize("source,kernel,at_least", [("paged_attention8.hip", "attention_", 14), ("paged_beams.hip", "select", 2)])
def test_a_workgroup_arrives_behind_its_stores(tmp_path, source, kernel, at_least):
    seen = 0
    for name, lines in listing(tmp_path, source).items():
        stores = [l for l in lines if re.match(r"(global|buffer|flat)_store.* sc1$", l)]
        counted = arrivals(lines)
        if not counted:
            assert not stores, name
            continue
        seen += 1
        assert kernel in name and stores, name
        for at, mine, others in counted:
            assert not mine and not others, (name, lines[at - 3:at + 1])
    assert seen >= at_least
