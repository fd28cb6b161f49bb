"""How products grouped by expert and those with 4-bit weights are launched (csrc/ffn_plan.h, compiled by itself): every size that a call takes fits a launch, and the
launch in tiles of several sizes has every output once."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
AT = 1 << 24                                           # an address at a multiple of 16
MOST = (1 << 31) - (1 << 16)                           # positions or rows of a descriptor
PLAIN, TOKENS, FEW, TILED = range(4)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = tmp_path_factory.mktemp("plan") / "ff_grouped_plan.so"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(path), os.path.join(HERE, "ff_grouped_plan.cpp")], check=True)
    return ctypes.CDLL(str(path))


def grouped(lib, rows, k, n, experts, gated=0, *, x_rows=None, index=0, x_stride=None, w_stride=None, expert_stride=None, x=0, w=0, w2=0, kernel=0):
    """(kernel, tile, whether the sizes are taken, threads of the launch, whether the planned one fits)"""
    w_stride = w_stride or k
    size = (ctypes.c_longlong * 11)(rows, x_rows or rows, k, n, experts, x_stride or k, w_stride, expert_stride or n * w_stride, AT + x, 2 * AT + w, 3 * AT + w2)
    out = (ctypes.c_ulonglong * 5)()
    lib.ff_grouped(size, gated, index, kernel, out)
    return tuple(out)


def s4(lib, rows, k, n, group, gated=0, *, x_stride=None, kernel=0):
    """(kernel, tile, whether the sizes are taken, threads of the launch)"""
    out = (ctypes.c_ulonglong * 4)()
    lib.ff_s4((ctypes.c_longlong * 5)(rows, k, n, x_stride or k, group), gated, kernel, out)
    return tuple(out)


ROWS = [1, 2, 15, 16, 17, 64, 65, 300, 1 << 13, (1 << 20) + 1, 1 << 25, (1 << 29) - 16385, 1 << 29, MOST]
WIDTHS = [1, 16, 17, 64, 129, 1000, 1 << 13, (1 << 17) + 1, 1 << 20, 1 << 22]


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("k", [1, 16, 1000, 4096, 16384, 40000, 131071])
def test_every_grouped_launch_fits(lib, gated, k):
    """fewer than 2^32 threads, of the library's choice and of every kernel that may be forced; the tiles' launches have no other kernel to fall back to"""
    taken = 0
    for rows, n, experts in itertools.product(ROWS, WIDTHS, (1, 2, 17, 64, 1000, 1024)):
        for forced in range(11):
            kernel, tile, fine, threads, fits = grouped(lib, rows, k, n, experts, gated, kernel=forced)
            if not fine:
                break
            taken += 1
            assert threads < 1 << 32 and (fits or kernel in (TOKENS, FEW)), (rows, n, experts, forced, kernel, tile, threads)
    assert taken > 1000


@pytest.mark.parametrize("gated", [0, 1])
def test_every_grouped_launch_of_drawn_sizes_fits(lib, gated):
    g = random.Random(gated)
    taken = 0
    for _ in range(20000):
        size = lambda most: min(most, int(2 ** g.uniform(0, most.bit_length())))  # noqa: E731
        rows, k, n, experts = size(MOST), size(131071), size(1 << 22), size(1024)
        call = dict(index=g.randrange(2), x_rows=size(MOST), x=g.choice((0, 0, 4, 1)), kernel=g.choice((0, 0, *range(1, 11))))
        kernel, tile, fine, threads, fits = grouped(lib, rows, k, n, experts, gated, **call)
        if fine:
            taken += 1
            assert threads < 1 << 32 and (fits or kernel in (TOKENS, FEW)), (rows, k, n, experts, call, kernel, tile, threads)
    assert taken > 5000


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("k", [1, 16, 2048, 4096, 8192, 16384, 32768, 131071])
def test_every_launch_with_4_bit_weights_fits(lib, gated, k):
    taken = 0
    for rows, n, group in itertools.product([*ROWS, 2, 3, 4, 5, 31, 32, 33, 64, 128], WIDTHS, (32, 64, 128, 256)):
        for forced in range(9):
            kernel, tile, fine, threads = s4(lib, rows, k, n, group, gated, kernel=forced)
            if not fine:
                break
            taken += 1
            assert threads < 1 << 32, (rows, n, group, forced, kernel, tile, threads)
    assert taken > 1000


def test_experts_at_odd_places_are_planned_as_what_their_copies_are(lib):
    """An expert's weights start at multiples of 16 bytes only if the stride between experts is one: else the copies go through registers, as of weights at such an address"""
    changed = 0
    for gated, rows, k, n in itertools.product((0, 1), (40, 100, 300, 600, 1000, 1500, 3000, 8000), (512, 1024, 4096, 8192), (512, 1024, 2048, 4096)):
        for off in (16, 8, 4, 2, 1):
            plan, moved, aligned = (grouped(lib, rows, k, n, 8, gated, **place)[:2] for place in (dict(expert_stride=n * k + off), dict(w=off), {}))
            assert plan == moved, (gated, rows, k, n, off)
            assert off != 16 or plan == aligned
            changed += plan != aligned
    assert changed > 20


def mixed(lib, offsets, rows, n, steps, gated, eighths):
    """(pieces of 64 x 128 that no workgroup has, that several have, workgroups outside, workgroups with something)"""
    out = (ctypes.c_longlong * 4)()
    lib.ff_mixed((ctypes.c_int * len(offsets))(*offsets), len(offsets) - 1, rows, n, steps, gated, eighths, out)
    return tuple(out)


KINDS = [(0, 0), (0, 1), (1, 0)]                       # (gated, eighths)


@pytest.mark.parametrize("gated,eighths", KINDS)
@pytest.mark.parametrize("n", [1, 128, 129, 300, 4096, 5461])
def test_tiles_of_several_sizes_have_every_output_once(lib, gated, eighths, n):
    g = random.Random(n)
    drawn = [[int(2 ** g.uniform(0, 11)) * g.choice((0, 1, 1)) for _ in range(g.randrange(1, 40))] for _ in range(40)]
    for counts in [[1], [0, 0], [256] * 7, [64], [65], [128], [129], [255], [257], [320], [321], [384], [385], [512, 0, 1], [1] * 300, [4096] * 8, [1024] * 32, *drawn]:
        for steps in (1, 8, 31, 32, 64, 1000):
            first, behind = g.choice(((0, 0), (5, 70)))
            offsets = [first]
            for c in counts:
                offsets.append(offsets[-1] + c)
            none, several, outside, some = mixed(lib, offsets, offsets[-1] + behind, n, steps, gated, eighths)
            assert (none, several, outside) == (0, 0, 0), (counts, steps, none, several, outside)
            assert (some > 0) == (sum(counts) > 0)


@pytest.mark.parametrize("gated,eighths", KINDS)
def test_offsets_that_are_none_give_no_tile_outside(lib, gated, eighths):
    g = random.Random(1)
    lists = [[0, 5, 3, 40], [-7, 10, 20, 99], [50, 40, 30, 20], [2 ** 31 - 1, -2 ** 31, 0, 40], [0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [0, 2 ** 31 - 1] * 512 + [0]]
    lists += [[g.choice((0, -5, 300, 2 ** 31 - 1, -2 ** 31, g.randrange(5000), g.randrange(-2000, 9000))) for _ in range(g.choice((2, 4, 9, 65, 1025)))] for _ in range(60)]
    for offsets in lists:
        for rows in (3, 40, 700, 5001):
            for n, steps in ((48, 1), (520, 40), (5000, 33)):
                assert mixed(lib, offsets, rows, n, steps, gated, eighths)[2] == 0, (offsets, rows, n, steps)
    # as many positions as there may be, and all of them every second expert's
    assert mixed(lib, [0, 2 ** 31 - 1] * 8 + [0], (1 << 29) - 16385, 16, 1, gated, eighths)[2] == 0
