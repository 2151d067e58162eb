"""Attention behind a shared prefix against its definition in 64 bits, with the tolerances of test_gpu_attention: keys are added up in
parts there too, and joining parts adds a rounding of 32 bits for each of at most 64, which (len + 64) * 2^-24 counts."""
import math

import pytest
import torch

import paper_2404_16109_amd as zk
from tests import serve_ref
from tests.test_gpu_attention import make
from tests.test_gpu_kvcache import arrays, device

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def share(table, shared):
    """The pages of the prefix, the table as the reference reads it (they begin every row), and as the call is given it."""
    front = table[0][:shared]
    full = [front + row[shared:] for row in table]
    given = [[-1] * min(shared, len(row)) + row[shared:] for row in table]
    return front, full, given


def call(cache, q, cu, lens, given, front, scale, max_new=None, max_len=None, **kw):
    new = [b - a for a, b in zip(cu, cu[1:])]
    pages = torch.tensor(front, dtype=torch.int32, device="cuda")
    return zk.kvcache_attention_prefix(cache, q, *device(cu, lens, given), pages, max_new or max(max(new), 1), max(lens) if max_len is None else max_len,
                                       scale, **kw)


def check(cache, q, cu, lens, table, shared, scale, **kw):
    front, full, given = share(table, shared)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, out, lse = call(cache, q, cu, lens, given, front, scale, fault=fault, **kw)
    assert rc == zk.ZK_OK
    torch.cuda.synchronize()
    assert fault.item() == 0
    want, wlse, size, score, weight = serve_ref.attention(*arrays(cache), q, cu, lens, full, scale)
    d, L = q.shape[2], max(lens)
    moved = (d + 16) * 2.0 ** -24 * score
    tol = (2.0 ** -11 + 2 * moved + (L + 64) * 2.0 ** -24)[..., None] * size + torch.finfo(q.dtype).eps / 2 * want.abs() + torch.finfo(q.dtype).tiny
    tol += (L * 127 * 2.0 ** -39 * weight)[..., None]
    assert torch.equal(out.isnan(), want.isnan()) and torch.equal(lse.isnan(), wlse.isnan())
    assert not (((out.double() - want).abs() > tol) & ~want.isnan()).any(), float((out.double() - want).abs().nan_to_num().max())
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and not out[empty].any()
    off = (lse.double() - wlse).abs()
    assert (off <= moved + (L + 64) * 2.0 ** -24 + 4 * 2.0 ** -24 * wlse.abs())[~empty & ~wlse.isnan()].all()
    return out, lse


CASES = [  # new, lens (with the prefix), heads, kv_heads, head_dim, page, pages of the prefix
    ([1], [17], 1, 1, 16, 16, 1), ([1, 1], [64, 65], 2, 1, 64, 64, 1), ([1, 1, 1], [65, 81, 200], 5, 1, 128, 16, 4), ([1, 1], [130, 190], 4, 2, 80, 32, 3),
    ([1, 1, 1, 1], [300, 320, 280, 257], 16, 4, 96, 16, 15), ([1] * 9, [513 + 7 * i for i in range(9)], 8, 8, 128, 128, 4), ([1] * 40, [700 + i for i in range(40)], 5, 1, 64, 64, 10),
    ([2, 0, 3], [140, 300, 150], 6, 3, 48, 32, 4), ([1, 1], [600, 530], 3, 1, 256, 256, 2), ([1, 2], [400, 420], 4, 4, 192, 16, 21),
    ([40, 1, 7], [600, 500, 520], 4, 2, 128, 64, 7), ([130, 33], [700, 333], 2, 1, 64, 32, 9), ([64, 64], [300, 999], 3, 3, 112, 16, 12),
    ([20], [300], 17, 1, 160, 32, 5), ([70, 2], [400, 400], 1, 1, 256, 128, 2), ([50, 50], [66, 100], 2, 2, 224, 16, 1), ([33], [2000], 1, 1, 32, 16, 100),
    ([1, 1], [3000, 2500], 4, 4, 128, 64, 38), ([1] * 3, [5000, 4999, 5100], 32, 2, 64, 16, 311),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("new,lens,heads,H,d,T,shared", CASES)
def test_prefix(dtype, new, lens, heads, H, d, T, shared):
    cache, q, cu, table, _ = make(zk, new, lens, heads, H, d, T, dtype, sum(lens) + d + heads)
    out, lse = check(cache, q, cu, lens, table, shared, d ** -0.5)
    front, full, given = share(table, shared)
    rc, again, alse = call(cache, q, cu, lens, given, front, d ** -0.5)   # sums come in one order
    assert torch.equal(again, out) and torch.equal(alse, lse)


@pytest.mark.parametrize("shared", [0, 1, 3, 4, 5, 20])
def test_where_the_prefix_ends(shared):
    """Pages of 16 in tiles of 64: ends inside a tile and on it, none, and all but a sequence's last tokens."""
    for new, lens in (([1, 1, 1], [321, 400, 321]), ([40, 3], [400, 330])):
        cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, 16, BF16, shared)
        check(cache, q, cu, lens, table, shared, 0.125)


@pytest.mark.parametrize("new,lens", [([10, 3], [200, 5]), ([1, 1, 1], [100, 64, 0]), ([300, 1], [256, 130]), ([50, 70], [256, 40]), ([2], [0])])
def test_rows_inside_the_prefix(new, lens):
    """The prompt itself, sequences that end within the prefix, rows before the first token: they see what their position allows."""
    for T, shared in ((16, 16), (64, 4), (128, 2)):
        longest = [max(x, 256) for x in lens]
        cache, q, cu, table, _ = make(zk, new, longest, 4, 2, 64, T, F16, 9)
        check(cache, q, cu, lens, table, shared, 0.125)


@pytest.mark.parametrize("new,lens", [([1, 1], [2500, 2300]), ([20, 1], [900, 800])])
def test_spread_as_the_caller_says(new, lens):
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, 16, F16, 3)
    for max_new, max_len in ((max(new), 1), (max(new), 10 ** 6), (max(new) + 7, lens[0]), (1000, 0)):
        check(cache, q, cu, lens, table, 30, 0.125, max_new=max_new, max_len=max_len)


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 260]), ([40, 2], [300, 260])])
@pytest.mark.parametrize("scale", [0.0, -0.1, 0.3, 1e-30])
def test_scales_of_scores(new, lens, scale):
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, 16, BF16, 31)
    check(cache, q, cu, lens, table, 12, scale)


@pytest.mark.parametrize("new", [[1, 1], [300, 300]])
def test_large_and_small_queries(new):
    lens, d = [700, 600], 128
    for size, kexp, scale in ((1e30, -40, 1e-25), (1e-30, 20, 1e20), (300.0, -6, 0.3)):
        cache, q, cu, table, gen = make(zk, new, lens, 4, 1, d, 32, BF16, 5)
        cache.k_exp.fill_(kexp)
        check(cache, (q.float() * size).to(BF16), cu, lens, table, 9, scale)


def test_many_rows_of_each_width():
    """Eight wavefronts to a workgroup up to 128 dimensions, four beyond; some without rows."""
    for d in (16, 64, 80, 128, 160):
        new, lens = [150, 3, 120, 1, 40], [500, 400, 330, 329, 400]
        cache, q, cu, table, _ = make(zk, new, lens, 8, 2, d, 32, F16, d)
        check(cache, q, cu, lens, table, 9, d ** -0.5)


def test_many_sequences():
    """More than a workgroup's threads, ragged, some without rows or tokens of their own."""
    g = torch.Generator().manual_seed(4)
    new = torch.randint(0, 3, (700,), generator=g).tolist()
    lens = (192 + torch.randint(0, 90, (700,), generator=g)).tolist()
    lens = [max(x, 192 + n) for x, n in zip(lens, new)]
    new[0], new[-1] = 2, 1
    cache, q, cu, table, _ = make(zk, new, lens, 6, 2, 32, 64, BF16, 4)
    check(cache, q, cu, lens, table, 3, 0.2)


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 260]), ([40, 2], [300, 260])])
def test_scales_far_apart(new, lens):
    """The prefix's values far above and far below the own ones: neither is lost beside the other."""
    d, T, shared = 64, 16, 15
    cache, q, cu, table, gen = make(zk, new, lens, 2, 1, d, T, F16, 5)
    cache.v.clamp_(-60, 60)
    for front_exp, own_exp in ((-40, 8), (8, -40), (-40, -40), (5, 8)):
        cache.v_exp.fill_(own_exp)
        cache.v_exp[table[0][:shared]] = front_exp
        _, full, given = share(table, shared)
        rc, out, lse = call(cache, q, cu, lens, given, table[0][:shared], d ** -0.5)
        want, wlse, size, score, weight = serve_ref.attention(*arrays(cache), q, cu, lens, full, d ** -0.5)
        moved = (d + 16) * 2.0 ** -24 * score
        assert ((lse.double() - wlse).abs() <= moved + (lens[0] + 64) * 2.0 ** -24 + 4 * 2.0 ** -24 * wlse.abs()).all()
        large = size.amax(-1, keepdim=True)
        tol = (2.0 ** -11 + 2 * moved + (lens[0] + 64) * 2.0 ** -24)[..., None] * size + 2.0 ** -11 * want.abs() + 2.0 ** -24 * large
        assert ((out.double() - want).abs() <= tol + 2.0 ** -24)[want.abs() < 60000].all()


@pytest.mark.parametrize("new,lens", [([1, 1, 1], [300, 260, 280]), ([40, 2, 33], [300, 260, 280])])
def test_not_finite(new, lens):
    """A poisoned page of the prefix reaches every row that sees it, one of a sequence's own that sequence, a query its row."""
    T, shared = 16, 15
    cache, q, cu, table, gen = make(zk, new, lens, 4, 2, 64, T, BF16, 7)
    front, full, given = share(table, shared)
    clean, clse = check(cache, q, cu, lens, table, shared, 0.125)
    cache.k_exp[front[3], 1] = zk.ZK_EXP_NAN
    out, _ = check(cache, q, cu, lens, table, shared, 0.125)
    assert out[:, 2:].isnan().all() and torch.equal(out[:, :2], clean[:, :2])
    cache.k_exp[front[3], 1] = -5
    clean, clse = check(cache, q, cu, lens, table, shared, 0.125)
    cache.v_exp[table[1][shared], 0] = zk.ZK_EXP_NAN
    rc, out, _ = call(cache, q, cu, lens, given, front, 0.125)
    assert out[cu[1]:cu[2], :2].isnan().all() and not out[:cu[1]].isnan().any() and not out[cu[2]:].isnan().any()
    cache.v_exp[table[1][shared], 0] = -5
    rc, clean, _ = call(cache, q, cu, lens, given, front, 0.125)
    q2 = q.clone()
    q2[0, 1, 5], q2[-1, 3, 63] = math.inf, math.nan
    rc, out, lse = call(cache, q2, cu, lens, given, front, 0.125)
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[-1, 3] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all() and torch.equal(out[~hit], clean[~hit])


def test_poisoned_pages_that_no_row_sees():
    """Rows inside the prefix: its later pages are not theirs.  Other pages of the cache are nobody's."""
    T, shared, new, lens = 16, 8, [3, 1], [20, 30]
    cache, q, cu, table, _ = make(zk, new, [128, 128], 4, 2, 64, T, BF16, 17)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    for page in range(cache.k.shape[0]):
        if page not in front[:2]:
            cache.k_exp[page] = cache.v_exp[page] = zk.ZK_EXP_NAN
    rc, out, lse = call(cache, q, cu, lens, given, front, 0.125)
    assert not want.isnan().any() and torch.equal(out, want) and torch.equal(lse, wlse)


@pytest.mark.parametrize("many", [False, True])
def test_what_the_device_refuses(many):
    new = [40, 2, 1] if many else [2, 2, 1]
    lens, T, shared = [300, 270, 290], 16, 16
    cache, q, cu, table, gen = make(zk, new, lens, 4, 2, 64, T, BF16, 9)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    for bad, what in (({"own": 10 ** 6}, zk.ZK_FAULT_PAGE), ({"own": -1}, zk.ZK_FAULT_PAGE), ({"front": 10 ** 6}, zk.ZK_FAULT_PAGE), ({"front": -1}, zk.ZK_FAULT_PAGE),
                      ({"len": 10 ** 6}, zk.ZK_FAULT_LENGTH), ({"len": -3}, zk.ZK_FAULT_LENGTH)):
        t2, l2, f2 = [list(r) for r in given], list(lens), list(front)
        if "own" in bad:
            t2[0][shared + 1] = bad["own"]
        elif "front" in bad:
            f2[5] = bad["front"]
        else:
            l2[0] = bad["len"]
        fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        rc, out, lse = call(cache, q, cu, l2, t2, f2, 0.125, max_len=300, fault=fault)
        assert rc == zk.ZK_OK and fault.item() == what, bad
        # the rows that would see a key in the page: those of the first sequence from position (shared + 1) * T on
        sees = max(0, (shared + 1) * T - (lens[0] - new[0])) if "own" in bad else 0
        hurt = slice(0, None) if "front" in bad else slice(sees, cu[1])
        assert out[hurt].isnan().all() and lse[hurt].isnan().all()
        assert torch.equal(out[:sees], want[:sees]) and torch.equal(lse[:sees], wlse[:sees])
        if "front" not in bad:
            assert torch.equal(out[cu[1]:], want[cu[1]:]) and torch.equal(lse[cu[1]:], wlse[cu[1]:])
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    pages = torch.tensor(front, dtype=torch.int32, device="cuda")
    rc, out, lse = zk.kvcache_attention_prefix(cache, q, *device([0, 10 ** 6, 5, 5], lens, given), pages, max(new), 300, 0.125, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH and out[5:].isnan().all()


def test_rows_behind_the_last_sequence():
    """Neither read nor written."""
    new, lens, T, shared = [1, 2], [200, 210], 16, 12
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, T, BF16, 19)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    more = torch.cat([q, torch.full((5, 4, 64), math.nan, dtype=BF16, device="cuda")])
    out, lse = torch.full_like(more, 3.0), torch.full((8, 4), 3.0, device="cuda")
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, _, _ = call(cache, more, cu, lens, given, front, 0.125, out=out, lse=lse, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == 0
    assert torch.equal(out[:3], want) and torch.equal(lse[:3], wlse) and out[3:].eq(3).all() and lse[3:].eq(3).all()


def test_strides():
    new, lens, d = [3, 1], [150, 190], 64
    cache, q, cu, table, gen = make(zk, new, lens, 4, 2, d, 16, BF16, 8)
    front, full, given = share(table, 9)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    wide = torch.zeros(4, 9, d + 3, dtype=BF16, device="cuda")
    wide[:, 1:9:2, 2:d + 2] = q
    out = torch.full((4, 5, d + 7), 3.0, dtype=BF16, device="cuda")
    rc, got, lse = call(cache, wide[:, 1:9:2, 2:d + 2], cu, lens, given, front, 0.125, out=out[:, 1:, 5:d + 5])
    assert rc == zk.ZK_OK and torch.equal(got, want) and torch.equal(lse, wlse)
    assert out[:, 0].eq(3).all() and out[:, :, :5].eq(3).all() and out[:, :, d + 5:].eq(3).all()


def test_as_the_attention_of_whole_tables():
    """The prefix's pages in every row of the table, read by kvcache_attention: the same to the roundings of two computations."""
    new, lens, T, shared = [1] * 12, [900 + 13 * i for i in range(12)], 64, 14
    cache, q, cu, table, _ = make(zk, new, lens, 20, 4, 128, T, BF16, 23)
    front, full, given = share(table, shared)
    rc, a, al = call(cache, q, cu, lens, given, front, 0.09)
    rc, b, bl = zk.kvcache_attention(cache, q, *device(cu, lens, full), 1, max(lens), 0.09)
    assert (al - bl).abs().max() < 1e-4 and (a.float() - b.float()).norm() <= 2.0 ** -7 * b.float().norm()


@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_streams_graphs_and_a_workspace_of_the_callers(new):
    """Captured once and replayed with other lengths, queries and pages; two graphs share a workspace, which holds anything."""
    lens, T, shared = [1000, 900], 64, 13
    cache, q, cu, table, gen = make(zk, new, lens, 4, 2, 128, T, BF16, 10)
    front, full, given = share(table, shared)
    args, pages = device(cu, lens, given), torch.tensor(front, dtype=torch.int32, device="cuda")
    need = zk.kvcache_attention_prefix_workspace_bytes(2, sum(new), max(new), 4, 2, 128, shared * T, 1000)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    assert zk.kvcache_attention_prefix(cache, q, *args, pages, max(new), 1000, 0.1, ws=ws[:need // 2])[0] == zk.ZK_E_BUFSZ
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        rc, want, wlse = zk.kvcache_attention_prefix(cache, q, *args, pages, max(new), 1000, 0.1, ws=ws)
        stream.synchronize()
        made = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                rc, out, lse = zk.kvcache_attention_prefix(cache, q, *args, pages, max(new), 1000, 0.1, ws=ws)
            made.append((graph, out, lse))
    for step in range(3):
        ws.fill_(0xff if step else 0)
        q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
        args[1].copy_(torch.tensor([1000 - step, 900 + step], dtype=torch.int32))
        for graph, out, lse in made:
            graph.replay()
        torch.cuda.synchronize()
        rc, again, alse = zk.kvcache_attention_prefix(cache, q, *args, pages, max(new), 1000, 0.1)
        for _, out, lse in made:
            assert torch.equal(out, again) and torch.equal(lse, alse)


def test_a_cache_beyond_32_bits():
    """Pages of the prefix whose codes lie more than 2^32 bytes into the cache."""
    H, d, T = 1, 256, 256
    pages = (1 << 32) // (T * d) + 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = zk.KvCache.empty(pages, H, T, d)
    table = [[pages - 1, 5, pages - 3], [pages - 1, 5, 7]]
    for b, L in enumerate((600, 520)):
        k, v = (torch.randn(L, H, d, generator=gen, device="cuda").to(BF16) for _ in range(2))
        assert zk.kvcache_append(cache, k, v, *device([0, L], [L], [table[b]]), L) == zk.ZK_OK
    for new in ([1, 1], [30, 8]):
        q = torch.randn(sum(new), 2, d, generator=gen, device="cuda").to(BF16)
        check(cache, q, [0, new[0], sum(new)], [600, 520], table, 2, 0.06)
