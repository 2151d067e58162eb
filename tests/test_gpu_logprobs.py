"""Log probabilities against their definition in 64 bits, at sizes where segments, chunks and ties can go wrong.

Tolerances.  A sum is of 32 terms to a thread, then six levels of lanes, four wavefronts and six levels of segments: 48
roundings at most, an exponential's argument is rounded to 2^-24 of its size, which the weights average to about the
entropy: 64 * 2^-24 * (1 + entropy) for lse, times (1 + entropy) again for the entropy; and what is near lse in size is
rounded once or twice to its own 2^-24."""
import math

import pytest
import torch

from tests import serve_ref

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    assert torch.cuda.is_available()
    return zk


def check(zk, x, targets, top):
    rc, got = zk.logprobs(x, targets, top)
    assert rc == zk.ZK_OK
    torch.cuda.synchronize()
    want = serve_ref.logprobs(x, targets.tolist(), top)
    for r in range(x.shape[0]):
        lse, ent = want["lse"][r], want["entropy"][r]
        fine = math.isfinite(lse)
        tol = 64 * STEP * (1 + ent) + 4 * STEP * abs(lse) if fine else 0.0

        def near(a, b, t):
            if math.isnan(b) or math.isinf(b):
                assert (math.isnan(a) and math.isnan(b)) or a == b, (r, a, b)
            else:
                assert abs(a - b) <= t + 4 * STEP * abs(b), (r, a, b, t)
        near(got["lse"][r].item(), lse, tol)
        near(got["entropy"][r].item(), ent, 64 * STEP * (1 + ent) ** 2 if fine else 0.0)
        near(got["target"][r].item(), want["target"][r], tol)
        if not math.isnan(lse):
            assert got["rank"][r].item() == want["rank"][r], r
        assert got["top_ids"][r].tolist() == want["top_ids"][r], r
        for a, b in zip(got["top"][r].tolist(), want["top"][r]):
            near(a, b, tol)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (2, 2, 2), (3, 5, 5), (1, 63, 32), (5, 255, 7), (2, 2047, 20), (3, 4099, 1),
                                            (2, 8193, 32), (700, 301, 3), (1, 33001, 5), (4, 70001, 8)])
def test_rows(zk, dtype, rows, vocab, top):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + vocab)
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 3).to(dtype)
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    targets[0] = vocab - 1
    check(zk, x, targets, top)


def test_long_vocabulary_and_its_limit(zk):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1, 1 << 19, generator=gen, device="cuda")
    check(zk, x, torch.tensor([77], dtype=torch.int32, device="cuda"), 32)
    rc, _ = zk.logprobs(torch.empty(1, (1 << 19) + 1, device="cuda"), None, 1)
    assert rc == zk.ZK_E_BADARG


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 5000, 20011])
def test_forbidden_tokens_and_ties(zk, dtype, vocab):
    """Rows that allow few tokens or none, masks of -inf and of the type's lowest value, rows of one value, many equal
    values at the top, both zeros, infinities and NaN."""
    low = torch.finfo(dtype).min
    x = torch.zeros(12, vocab, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    noise = torch.randn(vocab, generator=gen, device="cuda").to(dtype).float()
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, vocab // 2] = 3.0
    x[2] = low
    x[3] = low
    x[3, 5] = 1.0
    x[3, vocab - 1] = 1.0
    x[4] = 7.25
    x[5] = noise
    x[5, vocab // 3:] = 9.0
    x[6] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, 0.0, -0.0)
    x[7] = noise
    x[7, 3] = math.inf
    x[8] = noise
    x[8, vocab - 2] = math.nan
    x[9] = math.nan
    x[10] = noise
    x[10, 1:] = -math.inf
    x[11] = -noise.abs() - 60000.0 if dtype != torch.float16 else noise
    x = x.to(dtype)
    targets = torch.tensor([0, vocab // 2, 1, vocab - 1, vocab - 1, vocab - 1, vocab - 1, 3, 4, 0, 0, 7], dtype=torch.int32, device="cuda")
    check(zk, x, targets, 17)
    targets = torch.tensor([-1, vocab, 5, 4, 0, 0, 0, 4, -5, 1, 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    check(zk, x, targets, 1)


def test_strides_and_addresses(zk):
    """Rows that begin at every place of a 16-byte chunk, and are views of longer ones."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn(9, 3001, generator=gen, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        b = base.to(dtype)
        for off in (0, 1, 3, 6):
            x = b[1:, off:off + 2990]
            check(zk, x, torch.arange(8, dtype=torch.int32, device="cuda") * 300, 4)


def test_outputs_that_are_not_asked_for(zk):
    x = torch.randn(3, 1000, device="cuda")
    rc, got = zk.logprobs(x, None, 0)
    assert rc == zk.ZK_OK and got["target"] is None and got["top"].shape == (3, 0)
    assert torch.allclose(got["lse"].double(), torch.logsumexp(x.double(), 1), atol=1e-5)
    rc, _ = zk.logprobs(torch.empty(0, 1000, device="cuda"), None, 0)
    assert rc == zk.ZK_OK


def test_more_rows_than_a_grid_has(zk):
    x = torch.zeros(65540, 8, device="cuda")
    x[:, 3] = 1.0
    x[65539, 5] = 2.0
    rc, got = zk.logprobs(x, torch.full((65540,), 3, dtype=torch.int32, device="cuda"), 1)
    assert rc == zk.ZK_OK
    assert got["top_ids"][:65539].eq(3).all() and got["top_ids"][65539].item() == 5 and got["rank"][65539].item() == 1


def test_again_and_in_a_graph(zk):
    """The same bits on every run, on another stream and in a replayed graph."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(5, 30011, generator=gen, device="cuda")
    t = torch.randint(0, 30011, (5,), generator=gen, device="cuda", dtype=torch.int32)
    rc, first = zk.logprobs(x, t, 9)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        zk.logprobs(x, t, 9)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rc, other = zk.logprobs(x, t, 9)
    for _ in range(3):
        for v in other.values():
            v.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        rc, again = zk.logprobs(x, t, 9)
        torch.cuda.synchronize()
        for name in first:
            assert torch.equal(first[name], other[name]) and torch.equal(first[name], again[name])
