"""How attention behind a shared prefix is spread, on the host: every kernel has a batch that the GPU tests compute, and parts are whole, none of them empty, as
many as the join takes."""
import ctypes
import os
import random
import subprocess
import tempfile

import pytest

from tests.prefix_sizes import CASES, PAGE, SHARED, batch

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib():
    so = os.path.join(tempfile.mkdtemp(prefix="prefix_"), "prefix_plan_check.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "native", "prefix_plan_check.cpp"), "-o", so])
    return ctypes.CDLL(so)


def plan(lib, seqs, rows, most, kv_heads, head_dim, prefix, max_len):
    out = (ctypes.c_uint32 * 8)()
    lib.c_plan(seqs, ctypes.c_uint64(rows), ctypes.c_uint64(most), kv_heads, head_dim, prefix, max_len, out)
    return list(out)


@pytest.mark.parametrize("d,tiles,waves", CASES)
def test_batches_take_the_kernels_they_are_for(lib, d, tiles, waves):
    new, lens, group = batch(tiles, waves)
    p = plan(lib, len(new), sum(new) * group, max(new) * group, 2, d, SHARED * PAGE, max(lens))
    assert p[6:] == [tiles, waves] and p[2] > 0


def test_every_kernel_has_a_batch():
    assert {(-(-d // 32), tiles, waves) for d, tiles, waves in CASES} == {
        (dt, tiles, waves) for dt in range(1, 9) for tiles in (0, 1, 2) for waves in (4, 8) if waves == 4 or dt <= 4}


def test_parts(lib):
    rng = random.Random(3)
    for _ in range(20000):
        seqs, group, kv = int(2 ** rng.uniform(0, 15)), rng.choice([1, 2, 4, 5, 8, 17]), rng.choice([1, 2, 4, 8, 40])
        new = int(2 ** rng.uniform(0, 11))
        rows, d = rng.randint(new, seqs * new) * group, rng.choice(range(16, 257, 16))
        prefix, own = 16 * int(2 ** rng.uniform(0, 15)) * rng.randint(0, 1), int(2 ** rng.uniform(0, 16))
        row_tile, tiles, front, front_each, splits, each, _, waves = plan(lib, seqs, rows, new * group, kv, d, prefix, prefix + own)
        assert tiles == prefix // 64 and row_tile == 32 * waves
        assert front <= 32 and splits <= 32 and splits >= 1 and each >= 1
        if tiles:
            assert (front - 1) * front_each < tiles <= front * front_each
        else:
            assert front == 0
        mine = -(-(prefix + own - 64 * tiles) // 64)
        assert (splits - 1) * each < mine <= splits * each
