"""kvcache_attention_prefix through every kernel it has (held to the plan by test_prefix_plan.py): all sizes of a head, by one, two and many tiles
of rows to a sequence, with four and with eight wavefronts to a workgroup."""
import pytest
import torch

import paper_2404_16109_amd as zk
from tests.prefix_sizes import CASES, PAGE, SHARED, batch
from tests.test_gpu_attention import make
from tests.test_gpu_prefix import call, check, share

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,tiles,waves", CASES)
def test_kernels(d, tiles, waves):
    new, lens, group = batch(tiles, waves)
    dtype = torch.bfloat16 if (d // 16 + tiles) % 2 else torch.float16
    cache, q, cu, table, _ = make(zk, new, lens, 2 * group, 2, d, PAGE, dtype, d * 10 + tiles)
    out, lse = check(cache, q, cu, lens, table, SHARED, d ** -0.5)
    # parts shared out otherwise, and in whole: the same to the roundings
    front, full, given = share(table, SHARED)
    rc, again, alse = call(cache, q, cu, lens, given, front, d ** -0.5)
    assert rc == zk.ZK_OK and torch.equal(out, again) and torch.equal(lse, alse)
    check(cache, q, cu, lens, table, SHARED, d ** -0.5, max_len=4000)
    check(cache, q, cu, lens, table, 0, d ** -0.5)


@pytest.mark.parametrize("d,tiles,waves", [c for c in CASES if c[0] % 32 == 16 and c[1] == 2])
def test_masks_and_faults(d, tiles, waves):
    """Rows inside the prefix and before it, a page of the prefix that is none, and one that is poisoned, in the kernels of two tiles of rows."""
    new, lens, group = batch(tiles, waves)
    cache, q, cu, table, _ = make(zk, new, lens, 2 * group, 2, d, PAGE, torch.bfloat16, d)
    short = [max(n - 1, 0) if i % 3 == 0 else 40 + i for i, n in enumerate(new)]
    check(cache, q, cu, short, table, SHARED, d ** -0.5)
    front, full, given = share(table, SHARED)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, out, lse = call(cache, q, cu, lens, given, front[:3] + [-1] + front[4:], d ** -0.5, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_PAGE and out.isnan().all() and lse.isnan().all()
    cache.k_exp[front[8], 1] = zk.ZK_EXP_NAN
    out, _ = check(cache, q, cu, lens, table, SHARED, d ** -0.5)
    assert out[:, group:].isnan().all() and not out[:, :group].isnan().any()
