"""Products with 4-bit weights where a size, a value or a code is at its end."""
import math

import pytest
import torch

from tests import serve_ref
from tests.test_gpu_w4 import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    assert torch.cuda.is_available()
    return zk


# the last lengths whose scales fit a CU's LDS beside nothing else, the first that do not, and the longest
LONG = [(163840, 32), (163872, 32), (1 << 20, 32), (327680, 64), (327712, 64), (1 << 20, 64), (655360, 128), (655392, 128), (1 << 20, 128)]


@pytest.mark.parametrize("k,group", LONG)
@pytest.mark.parametrize("rows", [1, 3, 20])
def test_as_many_inputs_as_there_may_be(zk, rows, k, group):
    """Tolerance: as in test_gpu_w4 (its bound is relative to a group's sum of |x| and grows with the root of their number)."""
    n = 18
    gen, codes, scales = make(n, k, group, k // 32)
    w = serve_ref.weights(codes, scales, group)
    x = torch.randint(-32768, 32768, (rows, k), generator=gen, device="cuda", dtype=torch.int32).to(torch.int16)
    rc, y = zk.w4_matvec(x, codes, scales, group)
    assert rc == zk.ZK_OK
    # whole numbers: in halves of x whose products and sums stay below 2^53
    assert torch.equal(y, sum((part.double() @ w.double().t().contiguous()).long() << up for part, up in ((x.int() >> 8, 8), (x.int() & 255, 0))))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        xf = torch.randn(rows, k, generator=gen, device="cuda").to(dtype)
        unit = 2.0 ** -18
        rc, y = zk.w4_matvec(xf, codes, scales, group, unit)
        assert rc == zk.ZK_OK
        want = xf.double() @ w.double().t().contiguous() * unit
        groups = scales.shape[1]
        xa = torch.nn.functional.pad(xf.double().abs(), (0, groups * group - k)).reshape(rows, groups, group).sum(2)
        size = (xa[:, None, :] * scales.double()[None]).amax(2) * unit * math.sqrt(groups)
        tol = 8 * 2.0 ** -24 * 55 * size + torch.finfo(dtype).eps / 2 * want.abs() + torch.finfo(dtype).tiny
        assert ((y.double() - want).abs() <= tol).all()


def test_workspace_of_long_vectors(zk):
    """One size serves whatever outputs and groups a call has, and too little is told before anything runs."""
    k, group = 1 << 20, 32
    gen, codes, scales = make(4, k, group, 1)
    x = torch.randn(2, k, generator=gen, device="cuda").to(torch.bfloat16)
    need = zk.w4_matvec_workspace_bytes(torch.bfloat16, 2, k)
    rc, _ = zk.w4_matvec(x, codes, scales, group, ws=torch.empty(need // 4, dtype=torch.uint8, device="cuda"))
    assert rc == zk.ZK_E_BUFSZ
    rc, _ = zk.w4_matvec(x, codes, scales, group, ws=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert rc == zk.ZK_OK


def bound(x, codes, scales, group, unit):
    """test_gpu_w4's bound on the sums' error, elementwise: 8 * 2^-24 * 55 * unit * sqrt(groups) * max over groups of s * sum |x|."""
    k, groups = x.shape[1], scales.shape[1]
    xa = torch.nn.functional.pad(x.double().abs(), (0, groups * group - k)).reshape(x.shape[0], groups, group).sum(2)
    return 8 * 2.0 ** -24 * 55 * (xa[:, None, :] * scales.double()[None]).amax(2) * unit * math.sqrt(groups)


# rows and outputs that x in LDS, x laid out, and blocks of many columns have
WAYS = [(3, 40, 256), (5, 300, 2080), (6, 40, 320), (20, 500, 1056), (31, 8200, 416), (40, 9000, 320), (33, 16400, 288)]


@pytest.mark.parametrize("rows,n,k", WAYS)
def test_f32_beside_an_outlier(zk, rows, n, k):
    """One input far above the others that no output weighs: the others count with all their bits, in every number of vectors."""
    group, unit = 32, 2.0 ** -14
    gen, codes, scales = make(n, k, group, rows + n)
    scales[:, 1] = 0
    x = torch.randn(rows, k, generator=gen, device="cuda")
    x[:, 40] = 10.0 ** torch.linspace(4, 15, rows, device="cuda")
    rc, y = zk.w4_matvec(x, codes, scales, group, unit)
    assert rc == zk.ZK_OK
    want = x.double() @ (serve_ref.weights(codes, scales, group).double().t() * unit).contiguous()
    tol = bound(x, codes, scales, group, unit) + 2.0 ** -24 * want.abs()
    assert ((y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows,n,k", WAYS)
def test_rows_of_unlike_size(zk, rows, n, k):
    """Every row is as exact as if it stood alone: rows of 2^-80 and of 2^80, of zeros, of an infinity or a NaN side by side."""
    group, unit = 64, 2.0 ** -14
    gen, codes, scales = make(n, k, group, rows * n)
    size = torch.exp2(torch.randint(-80, 81, (rows, 1), generator=gen, device="cuda").float())
    base = torch.randn(rows, k, generator=gen, device="cuda")
    w = (serve_ref.weights(codes, scales, group).double().t() * unit).contiguous()
    for dtype in (torch.float32, torch.bfloat16):
        x = (base * size).to(dtype)
        x[rows // 2] = 0
        rc, y = zk.w4_matvec(x, codes, scales, group, unit)
        assert rc == zk.ZK_OK
        want = x.double() @ w
        tol = bound(x, codes, scales, group, unit) + torch.finfo(dtype).eps / 2 * want.abs()
        assert ((y.double() - want).abs() <= tol).all() and not y[rows // 2].any()
        hurt = x.clone()
        hurt[0, k - 1], hurt[rows - 1, 3] = math.nan, -math.inf
        if rows > 5:
            hurt[3, 100] = math.inf
        rc, z = zk.w4_matvec(hurt, codes, scales, group, unit)
        assert rc == zk.ZK_OK
        bad = torch.tensor([r for r in range(rows) if r in (0, rows - 1) or (r == 3 and rows > 5)], device="cuda")
        kept = torch.ones(rows, dtype=torch.bool, device="cuda")
        kept[bad] = False
        assert z[bad].isnan().all() and torch.equal(z[kept], y[kept])


@pytest.mark.parametrize("rows,n,k", WAYS)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_f32_weights_of_zero_cost_nothing(zk, rows, n, k, group):
    """Codes of zero add nothing, not even a rounding, however large the inputs they meet.  One weight to an output: x's parts
    times a code of 4 bits times a scale of 12 are exact, three of them are added and the unit is a power of two: 3 * 2^-24.
    None at all: zero."""
    unit = 2.0 ** -14
    gen, codes, scales = make(n, k, group, rows + n + group)
    at = torch.randint(0, k, (n,), generator=gen, device="cuda")
    c = torch.randint(-8, 8, (n,), generator=gen, device="cuda")
    c[::7] = 0
    nibbles = torch.full((n, k), 8, dtype=torch.int64, device="cuda")
    nibbles[torch.arange(n, device="cuda"), at] = c + 8
    codes = (nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)).to(torch.uint8)
    x = torch.rand(rows, k, generator=gen, device="cuda") * 5 + 1
    rc, y = zk.w4_matvec(x, codes, scales, group, unit)
    assert rc == zk.ZK_OK
    want = x.double() @ (serve_ref.weights(codes, scales, group).double().t() * unit).contiguous()
    assert ((y.double() - want).abs() <= 3 * 2.0 ** -24 * want.abs()).all()
    assert not y[:, ::7].any()


@pytest.mark.parametrize("rows,n", [(1, 64), (5, 64), (6, 64), (32, 64), (32, 8200), (17, 16400)])
def test_f32_of_few_weights(zk, rows, n):
    """Inputs of one sign, one weight in 64 not zero.  Relative to the sum of |w x|: four instructions of a group at two roundings
    of 2^-23 each, products with the scales and their sums in a wavefront (40 at most), wavefronts and parts (27): under 96 * 2^-24."""
    k, group, unit = 5120, 128, 2.0 ** -14
    gen, codes, scales = make(n, k, group, rows)
    keep = torch.rand(n, k, generator=gen, device="cuda") < 1 / 64
    nibbles = torch.where(keep, torch.randint(0, 16, (n, k), generator=gen, device="cuda"), 8)
    codes = (nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)).to(torch.uint8)
    x = torch.randn(rows, k, generator=gen, device="cuda") * 0.1 + 3
    rc, y = zk.w4_matvec(x, codes, scales, group, unit)
    assert rc == zk.ZK_OK
    w = (serve_ref.weights(codes, scales, group).double().t() * unit).contiguous()
    size = x.double() @ w.abs()
    assert ((y.double() - x.double() @ w).abs() <= 96 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("rows,n,k,group", [(1, 40, 4096, 128), (6, 40, 4096, 32), (40, 9000, 320, 64), (40, 16400, 288, 32), (2, 20, 1 << 20, 128),
                                            (20, 20, 1 << 20, 32)])
def test_as_large_as_x_may_be(zk, rows, n, k, group):
    """The largest bf16 below 2^88 by codes of one sign, -8 and 4: with 2^20 of them, what is summed comes nearest to 2^128.
    With scales of 2^11 every partial sum is 255 times a whole number of at most 2^20 / 32, times a power of two: 23 bits, so the
    result is exact in whatever order.  With scales of 4095 it is finite."""
    codes = torch.full((n, k // 2), 0xcc, dtype=torch.uint8, device="cuda")
    codes[1::2] = 0
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((rows, k), 255 * 2.0 ** 80, dtype=dtype, device="cuda")
        x[1::2] *= -1
        for scale in (2048, 4095):
            scales = torch.full((n, -(-k // group)), scale, dtype=torch.int16, device="cuda")
            rc, y = zk.w4_matvec(x, codes, scales, group, 2.0 ** -18)
            assert rc == zk.ZK_OK
            want = x.double() @ (serve_ref.weights(codes, scales, group).double().t() * 2.0 ** -18).contiguous()
            if scale == 2048:
                assert torch.equal(y, want.to(dtype))
            else:
                assert y.isfinite().all() and torch.equal(y.sign().double(), want.sign())


@pytest.mark.parametrize("n", [2559, 2560, 3001, 8191, 8192])
@pytest.mark.parametrize("rows", [10, 11, 21, 32, 33])
def test_f32_by_outputs_between(zk, rows, n):
    """Where calls change from blocks of five vectors to blocks of ten, and to all in one; tolerance as in test_gpu_w4."""
    for k, group in ((416, 32), (1056, 128)):
        unit = 2.0 ** -14
        gen, codes, scales = make(n, k, group, rows + n)
        x = torch.randn(rows, k, generator=gen, device="cuda")
        ws = torch.empty(zk.w4_matvec_workspace_bytes(torch.float32, rows, k), dtype=torch.uint8, device="cuda")
        rc, y = zk.w4_matvec(x, codes, scales, group, unit, ws=ws)
        assert rc == zk.ZK_OK
        want = x.double() @ (serve_ref.weights(codes, scales, group).double().t() * unit).contiguous()
        tol = bound(x, codes, scales, group, unit) + 2.0 ** -24 * want.abs()
        assert ((y.double() - want).abs() <= tol).all()
