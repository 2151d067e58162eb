"""Batches behind a shared prefix whose sequences are unlike: a prompt's next part beside single tokens, sequences without rows, rows that are
nobody's, sequences that are refused among others.  Each row's sums lie in a workspace by its place in the batch."""
import pytest
import torch

import paper_2404_16109_amd as zk
from tests.test_gpu_attention import make
from tests.test_gpu_kvcache import device
from tests.test_gpu_prefix import call, check, share

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16

BATCHES = [  # new, lens (with the prefix): the first prefix has 20 pages of 16
    ([300] + [1] * 40, [900] + [321 + 7 * i for i in range(40)]), ([1] * 70 + [129], [330 + i for i in range(70)] + [700]), ([1, 0, 257, 0, 0, 2, 33], [400, 350, 600, 330, 5, 322, 353]),
    ([0] * 130 + [5] + [0] * 130 + [40], [320] * 130 + [400] + [320] * 130 + [500]), ([17, 1, 32], [500, 900, 352]),
]


@pytest.mark.parametrize("new,lens", BATCHES)
@pytest.mark.parametrize("heads,H,d", [(4, 2, 64), (10, 2, 128), (1, 1, 256), (6, 3, 80)])
def test_unlike_sequences(new, lens, heads, H, d):
    cache, q, cu, table, _ = make(zk, new, lens, heads, H, d, 16, BF16, sum(lens) + d)
    check(cache, q, cu, lens, table, 20, d ** -0.5)


@pytest.mark.parametrize("new,lens", BATCHES[:3])
def test_a_workspace_of_just_the_size(new, lens):
    """Nothing beside it is written, what lay in it does not matter, and rows that are nobody's stay as they were."""
    T, shared, extra = 16, 20, 7
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, T, F16, 12)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    assert rc == zk.ZK_OK
    more = torch.cat([q, torch.full((extra, 4, 64), float("nan"), dtype=F16, device="cuda")])
    need = zk.kvcache_attention_prefix_workspace_bytes(len(new), more.shape[0], max(new), 4, 2, 64, shared * T, max(lens))
    space = torch.full((need + 8192,), 0xff, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(more, 3.0), torch.full((more.shape[0], 4), 3.0, device="cuda")
    rc, _, _ = call(cache, more, cu, lens, given, front, 0.125, out=out, lse=lse, ws=space[4096:4096 + need])
    assert rc == zk.ZK_OK
    assert space[:4096].eq(0xff).all() and space[4096 + need:].eq(0xff).all()
    assert torch.equal(out[:q.shape[0]], want) and torch.equal(lse[:q.shape[0]], wlse)
    assert out[q.shape[0]:].eq(3).all() and lse[q.shape[0]:].eq(3).all()


@pytest.mark.parametrize("many", [False, True])
def test_refused_sequences_among_others(many):
    """Too long, of a negative length, with more rows than were said: their rows are NaN and the fault is told, the others' are as without."""
    new = [3, 40, 2, 1, 2] if many else [3, 2, 2, 1, 2]
    lens, T, shared = [400, 380, 390, 350, 360], 16, 20
    cache, q, cu, table, _ = make(zk, new, lens, 4, 2, 64, T, BF16, 5)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.125)
    for b, bad in ((1, 10 ** 6), (4, -1), (0, 2 ** 31 - 1)):
        l2 = list(lens)
        l2[b] = bad
        fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        rc, out, lse = call(cache, q, cu, l2, given, front, 0.125, max_len=400, fault=fault)
        assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH
        hurt = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
        hurt[cu[b]:cu[b + 1]] = True
        assert out[hurt].isnan().all() and lse[hurt].isnan().all()
        assert torch.equal(out[~hurt], want[~hurt]) and torch.equal(lse[~hurt], wlse[~hurt])
    # a sequence without rows tells its fault too
    cu2, l2 = cu[:2] + cu[1:], lens[:1] + [-5] + lens[1:]
    g2 = given[:1] + given[:1] + given[1:]
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc, out, lse = call(cache, q, cu2, l2, g2, front, 0.125, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH and torch.equal(out, want) and torch.equal(lse, wlse)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    pages = torch.tensor(front, dtype=torch.int32, device="cuda")
    rc, out, lse = zk.kvcache_attention_prefix(cache, q, *device(cu, lens, given), pages, 2, 400, 0.125, fault=fault)
    long = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, n in enumerate(new):
        if n > 2:
            long[cu[b]:cu[b + 1]] = True
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH and out[long].isnan().all() and lse[long].isnan().all()
    assert not out[~long].isnan().any() and not lse[~long].isnan().any()


def test_a_part_of_a_prompt_beside_steps_takes_little():
    """2048 tokens of a prompt beside 127 single ones: the workspace is that of their rows, not of 128 times 2048 (286 MB)."""
    new = [2048] + [1] * 127
    lens = [4096] + [1100 + 3 * i for i in range(127)]
    T, shared, heads, H, d = 64, 16, 4, 2, 64
    cache, q, cu, table, _ = make(zk, new, lens, heads, H, d, T, BF16, 8)
    need = zk.kvcache_attention_prefix_workspace_bytes(128, sum(new), 2048, heads, H, d, shared * T, 4096)
    assert need < 32 << 20
    check(cache, q, cu, lens, table, shared, 0.125)


@pytest.mark.parametrize("seqs", [65, 130, 1000])
def test_many_sequences(seqs):
    """Steps of more sequences than are looked at at once: all alike, some without rows, one with most rows, rows behind them that are nobody's."""
    T, shared, d = 16, 4, 32
    for new in ([1] * seqs, [(i * 7) % 3 for i in range(seqs)], [0] * (seqs - 2) + [90, 1], [70] + [1] * (seqs - 1)):
        lens = [T * shared + n + (5 * i) % 40 for i, n in enumerate(new)]
        cache, q, cu, table, _ = make(zk, new, lens, 2, 1, d, T, F16, seqs)
        want, wlse = check(cache, q, cu, lens, table, shared, 0.2)
        front, full, given = share(table, shared)
        more = torch.cat([q, torch.full((300, 2, d), float("nan"), dtype=F16, device="cuda")])
        out, lse = torch.full_like(more, 3.0), torch.full((more.shape[0], 2), 3.0, device="cuda")
        fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        rc, _, _ = call(cache, more, cu, lens, given, front, 0.2, out=out, lse=lse, fault=fault)
        assert rc == zk.ZK_OK and fault.item() == 0
        assert torch.equal(out[:q.shape[0]], want) and torch.equal(lse[:q.shape[0]], wlse)
        assert out[q.shape[0]:].eq(3).all() and lse[q.shape[0]:].eq(3).all()


@pytest.mark.parametrize("at,value", [(70, 10 ** 6), (70, -5), (150, 10 ** 6), (10, -1), (199, 40)])
def test_many_sequences_of_which_one_is_refused(at, value):
    """One entry of cu is none: the two sequences that it bounds are skipped, and the fault is told; rows that no skipped one claims are as without."""
    seqs, T, shared, d = 200, 16, 4, 32
    new = [1] * seqs
    lens = [T * shared + 1 + i % 50 for i in range(seqs)]
    cache, q, cu, table, _ = make(zk, new, lens, 2, 1, d, T, BF16, 3)
    front, full, given = share(table, shared)
    rc, want, wlse = call(cache, q, cu, lens, given, front, 0.2)
    broken = list(cu)
    broken[at] = value
    claimed = torch.zeros(seqs, dtype=torch.bool, device="cuda")
    for b in (at - 1, at):
        lo, hi = max(broken[b], 0), min(broken[b + 1], seqs)
        if hi > lo:
            claimed[lo:hi] = True
    pages = torch.tensor(front, dtype=torch.int32, device="cuda")
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 3.0), torch.full((seqs, 2), 3.0, device="cuda")
    rc, _, _ = zk.kvcache_attention_prefix(cache, q, *device(broken, lens, given), pages, 1, max(lens), 0.2, out=out, lse=lse, fault=fault)
    assert rc == zk.ZK_OK and fault.item() == zk.ZK_FAULT_LENGTH
    mine = torch.ones(seqs, dtype=torch.bool, device="cuda")
    mine[at - 1:at + 1] = False     # rows of the sequences that are left
    sure = mine & ~claimed
    assert torch.equal(out[sure], want[sure]) and torch.equal(lse[sure], wlse[sure])
    only = claimed & ~mine
    assert out[only].isnan().all() and lse[only].isnan().all()
    both = claimed & mine
    assert (out[both].isnan() | (out[both] == want[both])).all()
