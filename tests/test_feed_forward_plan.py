"""How products of 8-bit rows are launched (csrc/ffn_plan.h, compiled by itself), against what the library asks of its callers."""
import ctypes
import itertools
import os
import subprocess

import pytest

from paper_2006_11735_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
AT = 1 << 24                                           # an address at a multiple of 16


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = tmp_path_factory.mktemp("plan") / "ff_plan.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(path), os.path.join(HERE, "ff_plan.cpp")], check=True)
    return ctypes.CDLL(str(path))


@pytest.fixture(scope="module")
def launch(lib):
    fn = lib.ff_launch
    fn.argtypes = [ctypes.POINTER(ctypes.c_longlong), ctypes.c_int, *[ctypes.c_size_t] * 3, *[ctypes.c_int] * 3, ctypes.POINTER(ctypes.c_ulonglong)]
    fn.restype = None

    def call(rows, k, n, gated, *, x=0, w=0, w2=0, x_stride=None, w_stride=None, workspace=True, kernel=0, split=0):
        """{kernel, tile, ranges, bytes} with x, w and w_up so many bytes behind a multiple of 16"""
        out = (ctypes.c_ulonglong * 4)()
        size = (ctypes.c_longlong * 5)(rows, k, n, x_stride or k, w_stride or k)
        fn(size, gated, AT + x, 2 * AT + w, 3 * AT + w2, workspace, kernel, split, out)
        return dict(zip(("kernel", "tile", "ranges", "bytes"), out))
    return call


def asked(rows, k, n, gated, x_stride=None, w_stride=None):
    d = B.linear_desc(rows=rows, k=k, n=n, x_stride=x_stride or k, w_stride=w_stride or k)
    return (B.igated_linear_s8_workspace_bytes if gated else B.ilinear_s8_workspace_bytes)(d)


PLACES = [dict(zip(("x", "w", "w2"), p)) for p in itertools.product((0, 1, 8), (0, 2, 4), (0, 1))]


@pytest.mark.parametrize("k,n", [(k, n) for k in (512, 2048, 4096, 8192, 11008, 16384) for n in (64, 256, 1024, 2048, 4096, 5000)] + [(1000, 301), (5461, 2048), (131071, 17)])
def test_no_launch_takes_more_workspace_than_is_asked_for(launch, k, n):
    """Whatever the operands' addresses are; and none that was asked of nothing splits k when it is handed another product's workspace."""
    for rows in (1, 4, 5, 8, 16, 17, 32, 40, 64, 65, 128, 200, 320, 512, 1000):
        for gated in (0, 1):
            size = asked(rows, k, n, gated)
            for place in PLACES:
                used = launch(rows, k, n, gated, **place)
                assert used["bytes"] <= size, (rows, k, n, gated, place, used, size)
                assert launch(rows, k, n, gated, workspace=False, **place)["bytes"] == 0


@pytest.mark.parametrize("pads", [(16, 0), (4, 16), (1, 0), (0, 3)])
def test_nor_with_strides_of_its_own(launch, pads):
    for rows, (k, n), gated in itertools.product((5, 24, 64, 100, 320), ((4096, 256), (8192, 1024), (11008, 2048), (4100, 300)), (0, 1)):
        strides = dict(x_stride=k + pads[0], w_stride=k + pads[1])
        for place in PLACES:
            assert launch(rows, k, n, gated, **strides, **place)["bytes"] <= asked(rows, k, n, gated, **strides)


@pytest.mark.parametrize("kernel,split", [(0, 1), (0, 2), (0, 16), (4, 0), (5, 3), (7, 16), (9, 0), (9, 16)])
def test_nor_under_a_tuning(launch, kernel, split):
    try:
        B.icnn_set_tuning("ff_kernel", kernel)
        B.icnn_set_tuning("ff_split", split)
        for rows, (k, n), gated in itertools.product((5, 24, 64, 100, 320), ((4096, 256), (8192, 1024), (11008, 2048), (1001, 90)), (0, 1)):
            size = asked(rows, k, n, gated)
            for place in PLACES:
                assert launch(rows, k, n, gated, kernel=kernel, split=split, **place)["bytes"] <= size
    finally:
        B.icnn_set_tuning("reset")


def test_the_sweep_reaches_launches_whose_plan_the_addresses_change(launch):
    plans = {tuple(launch(8, 11008, 1024, 0, x=x).values()) for x in (0, 1, 8)}
    assert len(plans) > 1 and any(p[2] > 1 for p in plans)


MOST = (1 << 31) - (1 << 16)                           # rows or outputs of a descriptor


def largest(lib, rows, k, n, gated, kernel=0):
    """(launches of a product, threads of the largest, its kernel)"""
    out = (ctypes.c_ulonglong * 3)()
    lib.ff_launches((ctypes.c_longlong * 5)(rows, k, n, k, k), gated, kernel, out)
    return tuple(out)


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("k", [1, 8, 16, 64, 1000, 8192, 16384, 40000])
def test_every_launch_fits(lib, k, gated):
    """fewer than 2^32 threads, whatever the sizes that a descriptor may have"""
    sizes = [1, 5, 64, 65, 300, 1 << 13, (1 << 20) + 1, (1 << 22) + 1, 1 << 23, 1 << 24, 1 << 28, 1 << 30, MOST]
    for rows, n in itertools.product(sizes, sizes):
        if rows * n <= 1 << 38:                        # (half a terabyte of results)
            count, threads, kernel = largest(lib, rows, k, n, gated)
            assert count >= 1 and threads < 1 << 32, (rows, n, count, threads, kernel)
            if rows * n <= 1 << 32 and n <= 1 << 22 and rows <= 1 << 26:
                assert count == 1, (rows, n)
            for forced in range(1, 10):
                assert largest(lib, rows, k, n, gated, forced)[1] < 1 << 32, (rows, n, forced)


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("rows,n", [(1, 1), (300, 5000), (MOST, 1), (1, MOST), (MOST, 65), ((1 << 27) + 300, 64), (3, (1 << 22) + 1), (1 << 18, 1 << 18), (100001, (1 << 22) + 70000)])
def test_ranges_cover_a_product_once(lib, rows, n, gated):
    out = (ctypes.c_longlong * 4096)()
    count = lib.ff_ranges((ctypes.c_longlong * 5)(rows, 16, n, 17, 19), gated, 1024, out)
    assert count >= 1
    parts = [tuple(out[4 * i:4 * i + 4]) for i in range(count)]
    assert sum(m * w for _, m, _, w in parts) == rows * n and all(m > 0 and w > 0 and m0 + m <= rows and n0 + w <= n for m0, m, n0, w in parts)
    columns = sorted({(n0, w) for _, _, n0, w in parts})
    lines = sorted({(m0, m) for m0, m, _, _ in parts})
    assert len(set(parts)) == count == len(columns) * len(lines)
    for spans, end in ((columns, n), (lines, rows)):
        at = 0
        for first, size in spans:
            assert first == at
            at += size
        assert at == end


def test_a_product_in_several_launches_asks_for_no_workspace():
    for rows, n in (((1 << 27) + 64, 64), (40, (1 << 22) + 64)):
        assert asked(rows, 16384, n, 0) == 0 and asked(rows, 16384, n, 1) == 0
