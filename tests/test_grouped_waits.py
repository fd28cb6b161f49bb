"""The counted waits of the kernels for products grouped by expert, and of the dense ones in tiles, from the built library.  A wave of the kernel for few rows that waits for its
turn's weights and rows leaves the next turn's in flight, so many copies and so many loads; one of a tile leaves the copies of all stages but the next.  So many must have
been issued behind those that it waits for: with fewer, some of these would be among those left."""
import re

import pytest

from code_util import kernels, loops


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return {k: kernels(tmp_path_factory.mktemp(k), k) for k in ("grouped_few_kernel", "grouped_tiled_kernel", "grouped_mixed_kernel", "linear_tiled_kernel")}


def copies_of(lines):
    return sum(s.startswith("buffer_load_dwordx4") and s.endswith("lds") for s in lines)


@pytest.mark.parametrize("rows", [1, 2, 4])
@pytest.mark.parametrize("gated", [0, 1])
def test_what_a_turn_s_wait_leaves_in_flight(code, rows, gated):
    names = [n for n in code["grouped_few_kernel"] if re.search(r"ILi%dELb%dELb1E" % (rows, gated), n)]
    assert len(names) == 1
    lines = code["grouped_few_kernel"][names[0]]
    copies, loads = 4 * (1 + gated), 4 * rows
    found = 0
    for at, s in enumerate(lines):
        m = re.match(r"s_waitcnt vmcnt\((\d+)\)$", s)
        ahead = next((q for q in lines[at + 1:at + 12] if q.startswith(("ds_read", "buffer_", "global_", "s_waitcnt vmcnt"))), "")
        if not m or int(m[1]) != copies + loads or not ahead.startswith("ds_read"):
            continue
        block = []
        for q in reversed(lines[:at]):
            if q.startswith(("label:", "s_cbranch", "s_branch")):
                break
            block.append(q)
        assert (copies_of(block), sum(q.startswith("global_load_dwordx4") for q in block)) == (copies, loads), (names[0], at)
        found += 1
    assert found == 2                                  # a pair of turns is the loop's body


def check_tile(name, body, stages, copies):
    """A step: half of a stage's copies, the wait, the barrier, half of the next one's"""
    at = body.index("s_barrier")
    waits = [i for i, s in enumerate(body) if "vmcnt" in s]
    assert body.count("s_barrier") == 1 and len(waits) == 1 and waits[0] < at, (name, waits, at)
    left = int(re.search(r"vmcnt\((\d+)\)", body[waits[0]])[1])
    parts = copies_of(body[:waits[0]]), copies_of(body[waits[0]:at]), copies_of(body[at:])
    assert left == (stages - 2) * copies and parts == (copies - copies // 2, 0, copies // 2), (name, left, parts)
    assert not any(s.startswith(("global_load", "global_store", "scratch_", "flat_")) for s in body), name


def steps_of(lines):
    return [b for b in loops(lines) if any("mfma" in s for s in b) and copies_of(b)]


@pytest.mark.parametrize("which", ["grouped_tiled_kernel", "linear_tiled_kernel"])
def test_what_a_step_s_wait_leaves_in_flight(code, which):
    seen = 0
    for name, lines in code[which].items():
        tn, tm, wn, wm, bk, stages, _gated, direct = (int(v) for v in re.search(which + "I" + r"L[ib](\d+)E" * 8, name).groups())
        bodies = steps_of(lines)
        assert len(bodies) == direct, name             # (through registers the compiler counts)
        for body in bodies:
            check_tile(name, body, stages, 32 * (tn * wn + tm * wm) * bk // 1024 // (wn * wm))
            seen += 1
    assert seen == 12                                  # six tiles, gated and not


def test_and_in_tiles_of_several_sizes(code):
    for name, lines in code["grouped_mixed_kernel"].items():
        _gated, direct, eighths = (int(v) for v in re.search("grouped_mixed_kernelI" + r"Lb(\d)E" * 3, name).groups())
        # products of a step, stages, copies of a wave
        sizes = {32: (2, 8), 16: (3, 6), 4: (6, 3)}
        found = []
        for body in steps_of(lines):
            products = sum("mfma" in s for s in body)
            check_tile(name, body, *sizes[products])
            found.append(products)
        assert sorted(found) == ([4] * eighths + [16, 32] if direct else []), name
