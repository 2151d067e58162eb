"""How products of 8-bit integers are spread, on the host: every way that some size takes has sizes that the GPU tests compute, and parts of k are
whole, none of them empty."""
import ctypes
import math
import os
import random
import subprocess
import tempfile

import pytest

from tests.i8_sizes import ALL, WAYS, name

HERE = os.path.dirname(os.path.abspath(__file__))
STEP, MOST_K = 128, 131056


@pytest.fixture(scope="module")
def lib():
    so = os.path.join(tempfile.mkdtemp(prefix="i8_"), "i8_plan_check.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "native", "i8_plan_check.cpp"), "-o", so])
    return ctypes.CDLL(so)


def plan(lib, rows, n, k):
    """(way, workgroups, parts of k, steps of a part)."""
    out, shape = (ctypes.c_uint32 * 5)(), (ctypes.c_uint32 * 2)()
    lib.c_plan(ctypes.c_size_t(rows), ctypes.c_size_t(n), ctypes.c_size_t(k), out)
    tile, nt, groups, splits, each = out
    if tile == 0:
        return ("few", 1 if rows <= 16 else 2, nt, splits > 1), groups, splits, each
    lib.c_tile(int(tile), shape)
    return ("%d x %d" % tuple(shape), 0, 0, splits > 1), groups, splits, each


@pytest.mark.parametrize("way,size", ALL, ids=lambda x: name(x) if isinstance(x[0], str) else "%d-%d-%d" % x)
def test_sizes_go_the_way_they_are_listed_under(lib, way, size):
    assert plan(lib, *size)[0] == way


def sizes(count):
    rng = random.Random(7)
    for _ in range(count):
        rows = rng.choice([1, rng.randint(2, 16), rng.randint(17, 32), int(33 * 2 ** rng.uniform(0, 13)), int(33 * 2 ** rng.uniform(0, 8))])
        n, k = int(2 ** rng.uniform(0, 17)), 16 * int(2 ** rng.uniform(0, math.log2(MOST_K // 16)))
        yield rows, n, k


def test_every_way_is_listed(lib):
    assert {plan(lib, *s)[0] for s in sizes(100000)} <= set(WAYS)


def test_parts(lib):
    for rows, n, k in sizes(20000):
        way, groups, splits, each = plan(lib, rows, n, k)
        steps = -(-k // STEP)
        assert groups > 0 and splits >= 1 and each % 2 == 0 and (splits - 1) * each < steps <= splits * each
        if way[0] == "few":
            assert groups == -(-n // (16 * way[2])) and splits <= 256
            assert splits == 1 or each >= 16
        else:
            r, o = map(int, way[0].split(" x "))
            assert groups == -(-rows // r) * -(-n // o) and splits <= 16
