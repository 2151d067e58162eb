"""Attention over the 8-bit cache at the smallest heads, with many rows: a tile has fewer pieces than the workgroup threads."""
import pytest
import torch

from tests.test_gpu_attention import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    assert torch.cuda.is_available()
    return zk


@pytest.mark.parametrize("new,lens,heads,H,d,T,window", [
    ([33], [33], 1, 1, 32, 16, 0), ([64], [64], 1, 1, 16, 64, 0), ([129], [700], 2, 1, 32, 16, 0), ([50, 3], [333, 200], 6, 3, 16, 32, 0),
    ([40], [1000], 4, 2, 32, 128, 100), ([200], [200], 1, 1, 16, 256, 7)])
def test_small_heads_of_many_rows(zk, new, lens, heads, H, d, T, window):
    for dtype in (torch.bfloat16, torch.float16):
        cache, q, cu, table, _ = make(zk, new, lens, heads, H, d, T, dtype, sum(lens) + d)
        check(zk, cache, q, cu, lens, table, d ** -0.5, window)
