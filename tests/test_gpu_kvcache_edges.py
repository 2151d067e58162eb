"""The cache of 8-bit keys and values at the ends of what a call may ask for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    assert torch.cuda.is_available()
    return zk


@pytest.mark.parametrize("tokens", [(1 << 20) - 1, (1 << 20) + 3, (1 << 24) + 5])
def test_more_tokens_than_a_launch_has_workgroups(zk, tokens):
    H, d, T = 1, 16, 256
    cache = zk.KvCache.empty(5, H, T, d)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(-127, 128, t.shape, generator=gen, device="cuda"))
    pages = torch.randint(0, 5, (-(-tokens // T),), generator=gen, device="cuda", dtype=torch.int32)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, k, v = zk.kvcache_read(cache, pages, tokens, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == 0
    for got, codes in ((k, cache.k[:, 0]), (v, cache.v[:, 0].transpose(1, 2).contiguous())):
        assert torch.equal(got.reshape(tokens, d), codes[pages.long()].reshape(-1, d)[:tokens].int())
    pages[-1] = -1
    rc, k, v = zk.kvcache_read(cache, pages, tokens, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_PAGE and not k[(tokens - 1) // T * T:].any() and not v[(tokens - 1) // T * T:].any()
