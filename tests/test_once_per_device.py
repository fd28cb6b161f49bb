"""A kernel's LDS limit is set once on each device that runs it (csrc/once_per_device.h, compiled by itself)."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def made(tmp_path_factory):
    path = tmp_path_factory.mktemp("once") / "once.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(path), os.path.join(HERE, "once_per_device.cpp")], check=True)
    lib = ctypes.CDLL(str(path))

    def call(pairs, fails=0):
        out = (ctypes.c_int * len(pairs))()
        lib.once_per_device((ctypes.c_longlong * len(pairs))(*[p[0] for p in pairs]), (ctypes.c_int * len(pairs))(*[p[1] for p in pairs]), len(pairs), fails, out)
        return list(out)
    return call


def test_each_device_has_its_own(made):
    assert made([(1, 0), (1, 0), (1, 1), (2, 1), (2, 0), (1, 1), (2, 1), (2, 0), (1, 0), (1, 7)]) == [1, 0, 1, 1, 1, 0, 0, 0, 0, 1]


def test_a_call_that_failed_is_made_again(made):
    assert made([(1, 0)] * 4, fails=2) == [1, 1, 1, 0]


def test_more_than_there_is_room_for_are_made_anew(made):
    pairs = [(i, 0) for i in range(1100)]
    assert made(pairs + pairs) == [1] * 1100 + [0] * 1024 + [1] * 76
