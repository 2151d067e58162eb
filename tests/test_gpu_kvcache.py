"""The cache of 8-bit keys and values: what an append leaves in it equals the definition bit for bit, whatever the sizes,
and what is read back can be proved to be in range."""
import math

import pytest
import torch

from tests import serve_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    assert torch.cuda.is_available()
    return zk


def paged(lens, T, seed, spare=2):
    """A table of distinct pages in a shuffled order; unused entries name no page."""
    used = [-(-max(x, 0) // T) for x in lens]
    order = torch.randperm(sum(used) + spare, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(max(used), 1)
    table, at = [], 0
    for u in used:
        table.append(order[at:at + u] + [-1] * (width - u))
        at += u
    return table, sum(used) + spare


def device(cu, lens, table):
    return [torch.tensor(t, dtype=torch.int32, device="cuda") for t in (cu, lens, table)]


def random_cache(zk, pages, H, T, d, gen):
    c = zk.KvCache.empty(pages, H, T, d)
    for t in (c.k, c.v):
        t.copy_(torch.randint(-127, 128, t.shape, generator=gen, device="cuda"))
    for t in (c.k_exp, c.v_exp):
        t.copy_(torch.randint(-12, 3, t.shape, generator=gen, device="cuda"))
    return c


def arrays(c):
    return [c.k, c.v, c.k_exp, c.v_exp]


CASES = [  # new tokens, lengths with them, heads, head_dim, page
    ([1], [1], 1, 16, 16), ([1], [17], 2, 64, 16), ([1, 1, 1], [64, 65, 100], 3, 128, 64), ([5], [5], 1, 80, 32),
    ([16], [40], 2, 96, 16), ([33, 0, 1], [33, 50, 7], 2, 48, 16), ([200], [300], 1, 256, 128), ([3, 130], [257, 200], 2, 112, 256),
    ([17, 15, 16, 1], [17, 31, 33, 48], 4, 32, 16), ([64, 63], [128, 127], 2, 128, 64), ([9], [6], 1, 64, 16), ([4, 2], [0, 1], 2, 32, 16),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("new,lens,H,d,T", CASES)
def test_append(zk, dtype, new, lens, H, d, T):
    seed = sum(new) * 31 + sum(lens) + d
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table, pages = paged(lens, T, seed)
    cu = [0] + torch.tensor(new).cumsum(0).tolist()
    cache = random_cache(zk, pages, H, T, d, gen)
    k, v = ((torch.randn(sum(new), H, d, generator=gen, device="cuda") *
             torch.exp2(torch.randint(-14, 8, (sum(new), H, 1), generator=gen, device="cuda").float())).to(dtype) for _ in range(2))
    want = serve_ref.append(*arrays(cache), k, v, cu, lens, table)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = device(cu, lens, table)
    assert zk.kvcache_append(cache, k, v, *args, max(new), fault=fault) == zk.ZK_OK
    assert fault.item() == 0
    for got, w in zip(arrays(cache), want):
        assert torch.equal(got, w)
    assert zk.kvcache_append(cache, k, v, *args, max(new)) == zk.ZK_OK      # again: nothing changes
    for got, w in zip(arrays(cache), want):
        assert torch.equal(got, w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_token_by_token(zk, dtype):
    """A page filled one token at a time, each larger or smaller than those before: exponents grow, codes are rounded again."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    H, d, T, L = 2, 64, 16, 37
    table, pages = paged([L], T, 1)
    cache = random_cache(zk, pages, H, T, d, gen)
    want = [t.clone() for t in arrays(cache)]
    for n in range(1, L + 1):
        k, v = ((torch.randn(1, H, d, generator=gen, device="cuda") * 2.0 ** ((n * 7) % 11 - 5)).to(dtype) for _ in range(2))
        want = serve_ref.append(*want, k, v, [0, 1], [n], table)
        assert zk.kvcache_append(cache, k, v, *device([0, 1], [n], table), 1) == zk.ZK_OK
    for got, w in zip(arrays(cache), want):
        assert torch.equal(got, w)


def test_sizes_at_the_ends(zk):
    """All zeros, the smallest and largest magnitudes, and the largest one for each exponent exactly."""
    H, d, T = 1, 16, 16
    rows = [0.0, 1e-45, 2.0 ** -41, 127 * 2.0 ** -40, 127.0, math.nextafter(127.0, 200.0), 127.00001, 63.5, 1.4e14, 3e38, 127 * 2.0 ** 40,
            254.0, 254.00002, 1.0, 0.75, 1e30]
    x = torch.tensor(rows, dtype=torch.float32, device="cuda")
    k = torch.stack([x, -x * 0.5] * 8, 1)[:, None, :].contiguous()
    n = len(rows)
    table = [[i] for i in range(n)]
    cu, lens = list(range(n + 1)), [1] * n
    cache = zk.KvCache.empty(n, H, T, d)
    want = serve_ref.append(*arrays(cache), k, -k, cu, lens, table)
    assert zk.kvcache_append(cache, k, -k, *device(cu, lens, table), 1) == zk.ZK_OK
    for got, w in zip(arrays(cache), want):
        assert torch.equal(got, w)
    assert cache.k_exp[0].item() == zk.ZK_EXP_MIN and cache.k_exp[9].item() == zk.ZK_EXP_MAX
    assert int(cache.k.max()) <= 127 and int(cache.k.min()) >= -127


def test_values_that_are_not_finite(zk):
    gen = torch.Generator(device="cuda").manual_seed(2)
    H, d, T = 3, 32, 16
    table, pages = paged([20, 20], T, 5)
    cache = random_cache(zk, pages, H, T, d, gen)
    k, v = (torch.randn(8, H, d, generator=gen, device="cuda") for _ in range(2))
    k[1, 0, 3], k[5, 2, 31], v[2, 1, 0] = math.nan, math.inf, -math.inf
    cu, lens = [0, 4, 8], [20, 18]
    want = serve_ref.append(*arrays(cache), k, v, cu, lens, table)
    assert zk.kvcache_append(cache, k, v, *device(cu, lens, table), 4) == zk.ZK_OK
    for got, w in zip(arrays(cache), want):
        assert torch.equal(got, w)
    assert (cache.k_exp == zk.ZK_EXP_NAN).sum() == 2 and (cache.v_exp == zk.ZK_EXP_NAN).sum() == 1
    # finite tokens afterwards do not hide it; a page that begins anew does
    k2 = torch.randn(1, H, d, generator=gen, device="cuda")
    before = cache.k_exp[table[0][1]].clone()
    assert zk.kvcache_append(cache, k2, k2, *device([0, 1, 1], [21, 18], table), 1) == zk.ZK_OK
    assert cache.k_exp[table[0][1], 0].item() == zk.ZK_EXP_NAN and before[0].item() == zk.ZK_EXP_NAN
    assert zk.kvcache_append(cache, k2, k2, *device([0, 1, 1], [17, 18], table), 1) == zk.ZK_OK
    assert cache.k_exp[table[0][1], 0].item() != zk.ZK_EXP_NAN


def test_strides(zk):
    """Heads side by side with others', rows of a wider projection, addresses that no wide load takes."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    H, d, T, n = 2, 48, 16, 21
    table, pages = paged([n + 3], T, 5)
    wide = torch.randn(n, 3, 2 * H + 1, d + 1, generator=gen, device="cuda").to(torch.bfloat16)
    for k, v in ((wide[:, 0, :H, :d], wide[:, 1, :H, 1:]), (wide[:, 0, 1:2 * H + 1:2, :d], wide[:, 2, :2 * H:2, :d]),
                 (wide[:, 0, :1, :d].expand(n, H, d), wide[:, 2, 1:2, :d].expand(n, H, d))):
        cache = random_cache(zk, pages, H, T, d, gen)
        want = serve_ref.append(*arrays(cache), k, v, [0, n], [n + 3], table)
        assert zk.kvcache_append(cache, k, v, *device([0, n], [n + 3], table), n) == zk.ZK_OK
        for got, w in zip(arrays(cache), want):
            assert torch.equal(got, w)


def test_what_the_device_refuses(zk):
    """Pages outside the cache and lengths that do not hold: nothing is written, the fault is told, the others go on."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    H, d, T = 2, 32, 16
    cache = random_cache(zk, 4, H, T, d, gen)
    before = [t.clone() for t in arrays(cache)]
    k = torch.randn(6, H, d, generator=gen, device="cuda")
    for table, cu, lens, want in (([[9], [1]], [0, 3, 6], [3, 3], zk.ZK_FAULT_PAGE), ([[-1], [1]], [0, 3, 6], [3, 3], zk.ZK_FAULT_PAGE),
                                  ([[0], [1]], [0, 3, 6], [17, 3], zk.ZK_FAULT_LENGTH), ([[0], [1]], [0, 3, 6], [-1, 3], zk.ZK_FAULT_LENGTH),
                                  ([[0], [1]], [4, 3, 6], [3, 3], zk.ZK_FAULT_LENGTH), ([[0], [1]], [-2, 3, 6], [3, 3], zk.ZK_FAULT_LENGTH)):
        for t, w in zip(arrays(cache), before):
            t.copy_(w)
        fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert zk.kvcache_append(cache, k, k, *device(cu, lens, table), 3, fault=fault) == zk.ZK_OK
        assert fault.item() == want
        only = serve_ref.append(*before, k, k, [3, 6], [3], [table[1]])
        for got, w in zip(arrays(cache), only):
            assert torch.equal(got, w)
    # a sequence with more rows than max_new, rows behind the call's
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert zk.kvcache_append(cache, k, k, *device([0, 6], [6], [[0]]), 5, fault=fault) == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH
    fault.zero_()
    assert zk.kvcache_append(cache, k, k, *device([0, 7], [7], [[0]]), 9, fault=fault) == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH


def test_codes_read_back_are_proved_in_range(zk):
    """kvcache_read gives the codes in order, and they go into the 8-bit range check as they are."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    H, d, T, L = 2, 64, 16, 32
    table, pages = paged([L], T, 9)
    cache = zk.KvCache.empty(pages, H, T, d)
    k, v = (torch.randn(L, H, d, generator=gen, device="cuda") for _ in range(2))
    args = device([0, L], [L], table)
    assert zk.kvcache_append(cache, k, v, *args, L) == zk.ZK_OK
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, kc, vc = zk.kvcache_read(cache, args[2][0], L, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == 0
    for h in range(H):
        for got, codes, exps, across, x in ((kc, cache.k, cache.k_exp, False, k), (vc, cache.v, cache.v_exp, True, v)):
            stands = serve_ref.numbers(codes, exps, table[0], h, across, L)
            scale = torch.exp2(exps[table[0], h].double()).repeat_interleave(T)[:L, None]
            assert torch.equal(got[:, h].double() * scale, stands)
            assert ((stands - x[:, h].double()).abs() <= scale / 2).all()
    tab = zk.Vec(256)
    assert zk.fr_from_i32(tab, torch.arange(-128, 128, dtype=torch.int32, device="cuda")) == 0
    X = kc.reshape(-1)
    rc, proof, _ = zk.tlookup_prove_small(bytes(32), X, None, None, X + 128, tab)
    assert rc == zk.ZK_OK and zk.tlookup_verify(bytes(32), proof, tab, X.numel())[0] == zk.ZK_OK
    rc, kc, vc = zk.kvcache_read(cache, torch.tensor([table[0][0], pages], dtype=torch.int32, device="cuda"), L, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_PAGE and kc[T:].eq(0).all() and vc[T:].eq(0).all()


def test_in_a_graph(zk):
    gen = torch.Generator(device="cuda").manual_seed(7)
    H, d, T = 2, 64, 16
    table, pages = paged([30, 9], T, 9)
    cache = random_cache(zk, pages, H, T, d, gen)
    before = [t.clone() for t in arrays(cache)]
    k = torch.randn(5, H, d, generator=gen, device="cuda")
    args = device([0, 3, 5], [30, 9], table)
    assert zk.kvcache_append(cache, k, k, *args, 3) == zk.ZK_OK
    want = [t.clone() for t in arrays(cache)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            assert zk.kvcache_append(cache, k, k, *args, 3) == zk.ZK_OK
    for _ in range(3):
        for t, w in zip(arrays(cache), before):
            t.copy_(w)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(arrays(cache), want):
            assert torch.equal(t, w)
