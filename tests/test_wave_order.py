"""Weights and scales that a wave's lanes put into LDS for each other, in the kernels for few rows: a turn's stores stand together, in front of its loads and behind those of the
turn before, in the built library (the hardware keeps a wave's order, and nothing else does)."""
import re

import pytest

from code_util import kernels, loops


@pytest.mark.parametrize("which,count,form", [("s4_few_kernel", 48, r"s4_few_kernel"), ("grouped_few_kernel", 6, r"ELb[01]ELb0E"), ("linear_few_kernel", 6, r"ELb[01]ELb0E")])
def test_a_turn_s_stores_and_loads(tmp_path, which, count, form):
    seen = set()
    for name, lines in kernels(tmp_path, which).items():
        if not re.search(form, name):
            continue                                   # (copied straight into LDS: its waits are counted)
        for body in loops(lines):
            kinds = [s[3] for s in body if s.startswith(("ds_read", "ds_write"))]
            if any("mfma" in s for s in body) and "w" in kinds:
                assert sum(a != b for a, b in zip(kinds, kinds[1:])) == 1, (name, "".join(kinds))
                seen.add(name)
    assert len(seen) == count
