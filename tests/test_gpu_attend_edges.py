"""Attention over the 8-bit cache at the smallest heads with many rows (a tile has fewer pieces than the workgroup threads), and
where the window has left pages behind."""
import pytest
import torch

from tests.test_gpu_attention import check, make
from tests.test_gpu_kvcache import device

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


@pytest.mark.parametrize("new,lens,window", [([1], [900], 100), ([3], [903], 100), ([1], [200], 5), ([60], [960], 100), ([60], [300], 17),
                                             ([200], [1000], 130), ([1] * 20, [1500 + 37 * i for i in range(20)], 1000),
                                             ([2] * 40, [2000 + 13 * i for i in range(40)], 1100), ([1], [6000], 5000)])
def test_pages_that_the_window_has_left(zk, new, lens, window):
    """A server frees what no row of the call can see any more: the table names no page there, and nothing is told or changed.
    The page that the first row's window begins in is needed: without it there is a fault, and that row is NaN."""
    T = 16
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, T, torch.bfloat16, len(lens) + window)
    args = device(cu, lens, table)
    rc, want, wlse = zk.kvcache_attention(cache, q, *args, max(new), max(lens), 0.125, window=window)
    assert rc == zk.ZK_OK
    left = [[-1 if (p + 1) * T <= max(lens[b] - new[b] - window + 1, 0) else page for p, page in enumerate(row)] for b, row in enumerate(table)]
    assert all(row.count(-1) > table[b].count(-1) for b, row in enumerate(left))
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, out, lse = zk.kvcache_attention(cache, q, *device(cu, lens, left), max(new), max(lens), 0.125, window=window, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == 0
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    left[0][(lens[0] - new[0] - window + 1) // T] = -1
    rc, out, lse = zk.kvcache_attention(cache, q, *device(cu, lens, left), max(new), max(lens), 0.125, window=window, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_PAGE
    assert out[0].isnan().all() and lse[0].isnan().all()
    hit = out.isnan().any(-1).any(-1)
    seen = torch.tensor([b == 0 and lens[0] - new[0] + i - window + 1 <= (lens[0] - new[0] - window + 1) // T * T + T - 1
                         for b in range(len(new)) for i in range(new[b])], device="cuda")
    assert torch.equal(hit, seen) and torch.equal(out[~hit], want[~hit])
