"""How the threads of the attention over many rows share out a tile of the cache, on the host: whatever the head's
dimension, every piece that a thread reads lies inside the tile (its run of 16 tokens indexes an array of four pages), and
those that are kept are each piece of the tile once."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
THREADS = 256


@pytest.fixture(scope="module")
def lib():
    so = os.path.join(tempfile.mkdtemp(prefix="attend_"), "attend_check.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "native", "attend_check.cpp"), "-o", so])
    return ctypes.CDLL(so)


@pytest.mark.parametrize("dt", range(1, 9))
def test_pieces_of_a_tile(lib, dt):
    rounds = (dt + 1) // 2
    out = np.zeros((rounds * THREADS, 6), dtype=np.uint32)
    lib.c_pieces(dt, THREADS, rounds, out.ctypes.data_as(ctypes.c_void_p))
    p, slot, c, dim, run, kept = out.T
    assert (p < 128 * dt).all() and (slot < 64).all() and (c < 2 * dt).all() and (dim < 32 * dt).all() and (run < 4).all()
    assert (slot // 16 < 4).all()
    mine = kept == 1
    assert sorted(p[mine]) == list(range(128 * dt))
    assert sorted(zip(slot[mine], c[mine])) == [(s, x) for s in range(64) for x in range(2 * dt)]
    assert sorted(zip(dim[mine], run[mine])) == [(d, r) for d in range(32 * dt) for r in range(4)]
