"""Products with 4-bit weights against their definition: whole numbers exactly, floats against 64 bits.

Tolerances.  A group's sum adds terms of at most 15.5 |x| and 12 |x| in 32 bits, twice: 2 * 27.5 * s * sum |x| at most.
What is added has random signs, so the roundings of a group, at most 2^-24 of that size each, add up as their root: 16
instructions of a group each round once or twice and keep what they add up inside exact; the groups and eight wavefronts
add 2^-24 of the result's parts.  As a bound that leaves no room for a missing term: 8 * 2^-24 * 55 * unit * max over
groups of s * sum |x| * sqrt(groups), and half a step of the result's type."""
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


def make(n, k, group, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.randint(0, 4096, (n, -(-k // group)), generator=gen, device="cuda", dtype=torch.int16)
    return gen, codes, scales


SHAPES = [(1, 1, 32, 32), (1, 17, 64, 128), (2, 16, 160, 128), (3, 100, 96, 64), (5, 33, 1024, 32), (6, 31, 1056, 128), (8, 48, 2080, 64),
          (9, 15, 4128, 32), (16, 129, 512, 128), (17, 64, 1312, 64), (33, 20, 17440, 128), (70, 65, 544, 32), (1, 5000, 64, 64),
          (40, 300, 2048, 128), (130, 257, 1184, 64),
          # many outputs: two, four and six tiles of columns, 64 and 128 outputs to a workgroup, one to five chunks of inputs
          (17, 8200, 160, 64), (31, 8199, 544, 32), (32, 9000, 1056, 128), (18, 16500, 416, 64), (25, 16390, 544, 128), (60, 8193, 672, 64),
          (33, 16400, 96, 32), (50, 16450, 1184, 128), (90, 8200, 288, 64), (70, 16385, 672, 32)]


@pytest.mark.parametrize("rows,n,k,group", SHAPES)
def test_integers_exactly(zk, rows, n, k, group):
    gen, codes, scales = make(n, k, group, rows + k)
    x = torch.randint(-32768, 32768, (rows, k), generator=gen, device="cuda", dtype=torch.int32).to(torch.int16)
    x[0, 0], x[-1, -1] = -32768, 32767
    rc, y = zk.w4_matvec(x, codes, scales, group)
    assert rc == zk.ZK_OK
    want = x.long().cpu() @ serve_ref.weights(codes, scales, group).t().cpu()
    assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,n,k,group", SHAPES)
def test_floats(zk, dtype, rows, n, k, group):
    gen, codes, scales = make(n, k, group, rows + k + 1)
    x = torch.randn(rows, k, generator=gen, device="cuda").to(dtype)
    unit = 2.0 ** -14
    rc, y = zk.w4_matvec(x, codes, scales, group, unit)
    assert rc == zk.ZK_OK
    w = serve_ref.weights(codes, scales, group).double()
    want = x.double() @ w.t().contiguous() * unit
    groups = scales.shape[1]
    xa = torch.nn.functional.pad(x.double().abs(), (0, groups * group - k)).reshape(rows, groups, group).sum(2)
    size = (xa[:, None, :] * scales.double()[None]).amax(2) * unit * math.sqrt(groups)
    tol = 8 * 2.0 ** -24 * 55 * size + torch.finfo(dtype).eps / 2 * want.abs() + torch.finfo(dtype).tiny
    assert ((y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 9), (torch.float16, 3), (torch.bfloat16, 3)])
def test_every_code_and_place(zk, dtype, bits):
    """One input after the other set, whole numbers that every step holds exactly."""
    n, k, group = 40, 256, 64
    gen, codes, scales = make(n, k, group, 9)
    scales %= 4
    w = serve_ref.weights(codes, scales, group)
    x = torch.diag(torch.arange(1, k + 1, device="cuda") % (1 << bits)).to(dtype)
    rc, y = zk.w4_matvec(x, codes, scales, group, 1.0)
    assert rc == zk.ZK_OK
    assert torch.equal(y.double(), x.double() @ w.double().t().contiguous())


def test_f32_keeps_its_bits(zk):
    """x of 24 bits by single weights: the three parts add up to x itself."""
    n, k, group = 16, 32, 32
    codes = torch.full((n, k // 2), 0x88, dtype=torch.uint8, device="cuda")
    for i in range(n):
        codes[i, i] = 0x89                                   # weight 1 at input 2i
    scales = torch.ones(n, 1, dtype=torch.int16, device="cuda")
    for size in (1.0, 2.0 ** -60, 2.0 ** 60):
        x = (torch.rand(1, k, device="cuda") + 1.0) * size
        rc, y = zk.w4_matvec(x, codes, scales, group, 1.0)
        assert rc == zk.ZK_OK
        # the constant that the codes are shifted by costs sums of 32 inputs their last bits
        assert ((y[0] - x[0, ::2]).abs() <= 8 * 2.0 ** -24 * 55 * 64 * size).all()
        one = torch.zeros_like(x)
        one[0, 6] = x[0, 6]
        rc, y = zk.w4_matvec(one, codes, scales, group, 1.0)
        assert abs(y[0, 3].item() - x[0, 6].item()) <= 2 * 2.0 ** -23 * 12 * x[0, 6].item() and y[0, 2].item() == 0.0


def test_not_finite(zk):
    gen, codes, scales = make(64, 256, 128, 4)
    x = torch.randn(5, 256, generator=gen, device="cuda")
    clean = x.clone()
    x[1, 7], x[3, 200] = math.inf, math.nan
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        rc, y = zk.w4_matvec(x.to(dtype), codes, scales, 128, 2.0 ** -12)
        rc2, z = zk.w4_matvec(clean.to(dtype), codes, scales, 128, 2.0 ** -12)
        assert rc == rc2 == zk.ZK_OK
        assert y[[1, 3]].isnan().all() and torch.equal(y[[0, 2, 4]], z[[0, 2, 4]])


def test_strides_outputs_and_streams(zk):
    gen, codes, scales = make(100, 320, 64, 6)
    wide = torch.randn(20, 400, generator=gen, device="cuda").to(torch.bfloat16)
    x = wide[::2, 8:328]
    rc, want = zk.w4_matvec(x.contiguous(), codes, scales, 64, 2.0 ** -12)
    out = torch.full((10, 130), 5.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        rc, y = zk.w4_matvec(x, codes, scales, 64, 2.0 ** -12, out=out[:, 7:107])
    s.synchronize()
    assert rc == zk.ZK_OK and torch.equal(y, want)
    assert out[:, :7].eq(5).all() and out[:, 107:].eq(5).all()


def test_expanded_weights_prove(zk):
    """The integers that come out are the Y of the matmul proof for the integers that went in."""
    rows, n, k, group = 5, 24, 64, 32
    gen, codes, scales = make(n, k, group, 12)
    x = torch.randint(-3000, 3000, (rows, k), generator=gen, device="cuda", dtype=torch.int32).to(torch.int16)
    rc, W = zk.w4_expand_i16(codes, scales, group)
    assert rc == zk.ZK_OK and torch.equal(W.long().t(), serve_ref.weights(codes, scales, group))
    rc, y = zk.w4_matvec(x, codes, scales, group)
    seed = bytes(range(32))
    rc, proof = zk.matmul_sumcheck_prove_i16(seed, x, W)
    assert rc == zk.ZK_OK

    def vec(t):
        v = zk.Vec(t.numel())
        assert zk.fr_from_i32(v, t.reshape(-1).to(torch.int32).contiguous()) == 0
        return v
    assert y.abs().max() < 2 ** 31
    assert zk.matmul_sumcheck_verify(seed, proof, rows, k, n, Y=vec(y), X=vec(x), W=vec(W)) == zk.ZK_OK
    y[3, 5] += 1
    assert zk.matmul_sumcheck_verify(seed, proof, rows, k, n, Y=vec(y), X=vec(x), W=vec(W)) == zk.ZK_E_REJECT


def test_in_a_graph(zk):
    gen, codes, scales = make(500, 1024, 128, 2)
    x = torch.randn(40, 1024, generator=gen, device="cuda")
    rc, want = zk.w4_matvec(x, codes, scales, 128, 0.01)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rc, y = zk.w4_matvec(x, codes, scales, 128, 0.01)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        rc, again = zk.w4_matvec(x, codes, scales, 128, 0.01)
        assert torch.equal(y, want) and torch.equal(again, want)
