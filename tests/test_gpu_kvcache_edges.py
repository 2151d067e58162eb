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


@pytest.mark.parametrize("tokens,d", [((1 << 24) + 7, 16), ((1 << 28) + 5, 80)])
def test_more_pages_than_a_launch_has_workgroups(zk, tokens, d):
    """One key and one value, again and again: every slot of every page has their codes, and what is behind the end is cleared."""
    H, T = 1, 16
    pages = -(-tokens // T)
    cache = zk.KvCache.empty(pages, H, T, d)
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(1, H, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, tokens], [tokens])]
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert zk.kvcache_append(cache, k.expand(tokens, H, d), v.expand(tokens, H, d), *args, table, tokens, fault=fault) == zk.ZK_OK
    assert fault.item() == 0
    one = zk.KvCache.empty(1, H, T, d)
    first = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, T], [T], [[0]])]
    assert zk.kvcache_append(one, k.expand(T, H, d), v.expand(T, H, d), *first, T) == zk.ZK_OK
    assert one.k.any() and one.v.any()
    for got, want in ((cache.k, one.k), (cache.v, one.v), (cache.k_exp, one.k_exp), (cache.v_exp, one.v_exp)):
        for at in range(1, pages, 1 << 21):                 # page 0 is the last, and not full
            assert bool((got[at:at + (1 << 21)] == want).all())
    left = tokens % T
    assert torch.equal(cache.k[0, 0, :left], one.k[0, 0, :left]) and not cache.k[0, 0, left:].any()
    assert torch.equal(cache.v[0, 0, :, :left], one.v[0, 0, :, :left]) and not cache.v[0, 0, :, left:].any()
