"""The statistics of block_norm where 64 bits are not enough to add up a row in any order: means of squares whose 1 / sqrt lies next to the middle
between two numbers of 32 bits, and means that cancel.  The sum is that of the definition, exact and rounded once (rational numbers
here): a row's codes, scales and values are the same alone, in a batch, and at any address."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2404_16109_amd as zk
from tests import layer_ref as ref
from tests.test_gpu_norm import same, strided

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = float(np.float32(1e-5))


def down(value, dtype):
    """The largest number of the type that is not above `value` (a positive rational)."""
    t = torch.tensor(float(value), dtype=torch.float64).to(dtype)
    while Fraction(float(t)) > value:
        t = torch.nextafter(t.float(), torch.tensor(0.0)).to(dtype) if dtype == F32 else (t.view(torch.int16) - 1).view(dtype)
    return t


def row_near_a_middle(dim, dtype, off, pairs, gen):
    """A row whose mean of squares puts 1 / sqrt(mean + eps) within some units of 2^-53 of the middle between two floats, `off` of them
    aside; with `pairs` every number has its negative, so that the mean is 0."""
    free = 12                                  # numbers that bring the sum where it shall be
    half = dim // 2 if pairs else dim
    x = torch.randn(half, generator=gen) * torch.exp2(-torch.randint(0, 7, (half,), generator=gen).float())
    x = x.to(dtype)
    x[-free:] = 0
    times = 2 if pairs else 1
    have = times * sum(Fraction(v) ** 2 for v in x.double().tolist())
    eps = Fraction(EPS)
    f = np.float32(1 / math.sqrt(float(have * (1 + Fraction(1, 1 << 21)) / dim + eps)))
    middle = (Fraction(float(f)) + Fraction(float(np.nextafter(f, np.float32(0))))) / 2
    wanted = dim * (1 / middle ** 2 - eps) * (1 + Fraction(off, 1 << 53))
    left = (wanted - have) / times
    assert left > 0
    for i in range(half - free, half):
        root = Fraction(math.isqrt(int(left * (1 << 240)))) / (1 << 120)
        if root < Fraction(1, 1 << 24) and dtype == F16:
            break
        x[i] = down(root, dtype)
        left -= Fraction(float(x[i])) ** 2
    assert abs(left * times / wanted) < Fraction(1, 1 << 54)
    if pairs:
        x = torch.cat([x, -x, x.new_zeros(dim - 2 * half)])
    return x[torch.randperm(dim, generator=gen)]


def rstd_of(row, mean=0.0):
    squares = sum((Fraction(v) - Fraction(mean)) ** 2 for v in row.double().tolist())
    return np.float32(1.0 / math.sqrt(float(squares) / len(row) + EPS))


def rows_of(dim, dtype, pairs, count=16):
    gen = torch.Generator().manual_seed(dim * 3 + pairs)
    rows = torch.stack([row_near_a_middle(dim, dtype, i - count // 2, pairs, gen) for i in range(count)])
    rstd = torch.from_numpy(np.array([rstd_of(r) for r in rows]))
    return rows, rows.float() * rstd[:, None]          # the mean is 0 where one is taken off


def look(rows, h, norm, batch):
    """Alone, in a batch and at odd addresses."""
    codes, scales = ref.codes_of(h)
    count, dim = rows.shape
    many = rows.repeat(-(-batch // count), 1)
    for x in (rows[:1], rows, many, strided(rows, 3, 1)[0], strided(many, 1, 1)[0]):
        x = x.cuda()
        n = x.shape[0]
        rc, _, got, got_scales = zk.block_norm(x, norm=norm, eps=EPS, quantise=True)
        assert rc == zk.ZK_OK
        at = torch.arange(n) % count
        same(got_scales, scales[at])
        same(got, codes[at])
        rc, _, got, _ = zk.block_norm(x, norm=norm, eps=EPS)
        assert rc == zk.ZK_OK
        same(got, h[at].to(rows.dtype))


@pytest.mark.parametrize("dtype,dim", [(F32, 520), (F32, 4100), (F32, 8200), (F16, 1024), (F16, 5120), (BF16, 1032), (BF16, 4096), (BF16, 8200), (BF16, 1001)])
def test_squares(dtype, dim):
    look(*rows_of(dim, dtype, False), zk.ZK_NORM_RMS, 1024)


@pytest.mark.parametrize("dtype,dim", [(F32, 260), (F32, 4097), (F16, 1024), (BF16, 2048), (BF16, 1001)])
def test_around_a_mean_of_zero(dtype, dim):
    look(*rows_of(dim, dtype, True), zk.ZK_NORM_LAYER, 1024)


@pytest.mark.parametrize("dtype,dim", [(F32, 20000), (BF16, 16385), (F32, 32768)])
def test_rows_in_lds(dtype, dim):
    look(*rows_of(dim, dtype, False, 4), zk.ZK_NORM_RMS, 8)
    look(*rows_of(dim, dtype, True, 4), zk.ZK_NORM_LAYER, 8)


@pytest.mark.parametrize("dim", [256, 1023, 8196, 20000])
def test_means_next_to_the_middle(dim):
    """Sums that cancel down to the middle between two floats, and beside it; the variance is taken around the mean in 64 bits."""
    gen = torch.Generator().manual_seed(dim)
    rows, want = [], []
    for off in range(-4, 5):
        half = (dim - 8) // 2
        a = torch.randn(half, generator=gen) * torch.exp2(torch.randint(-12, 13, (half,), generator=gen).float())
        mean = np.float32(1.3 + off / 64)
        middle = (Fraction(float(mean)) + Fraction(float(np.nextafter(mean, np.float32(9))))) / 2
        left = dim * middle * (1 + Fraction(off, 1 << 53))
        rest = torch.zeros(dim - 2 * half)
        for i in range(len(rest)):
            rest[i] = float(left)
            left -= Fraction(float(rest[i]))
        x = torch.cat([a, -a, rest])[torch.randperm(dim, generator=gen)]
        m = float(sum(Fraction(v) for v in x.tolist())) / dim
        rows.append(x)
        want.append((x - torch.tensor(np.float32(m))) * torch.tensor(rstd_of(x, m)))
    look(torch.stack(rows), torch.stack(want), zk.ZK_NORM_LAYER, 16)


def test_a_block_in_between():
    """The norm behind a block and that of the residual stream, each next to a middle."""
    z, t = rows_of(1024, F32, False)
    for batch in (1, 16, 1024):
        zb = z.repeat(-(-batch // 16), 1)[:batch].cuda()
        x = torch.zeros_like(zb)
        rc, r, _, _ = zk.block_norm(x, zb, norm=zk.ZK_NORM_NONE, post_norm=zk.ZK_NORM_RMS, eps=EPS)
        assert rc == zk.ZK_OK
        same(r, t.repeat(-(-batch // 16), 1)[:batch])


@pytest.mark.parametrize("dim", [64, 1021, 8196, 32768])
def test_means_of_any_size(dim):
    """Numbers from the largest to the smallest, whose sum is anything, of either sign, and zero."""
    gen = torch.Generator().manual_seed(dim)
    half = dim // 2
    sizes = ((-100, 120), (-149, -120), (100, 127), (-20, 0))
    rows, want = [], []
    for i, (lo, hi) in enumerate(sizes * 2):
        a = (torch.rand(half, generator=gen) + 0.5) * torch.exp2(torch.randint(lo, hi, (half,), generator=gen).double()).float()
        a *= torch.randint(0, 2, (half,), generator=gen) * 2 - 1
        b = a.flip(0)
        x = torch.cat([a, -b if i >= 4 else b * 0.7, a.new_zeros(dim - 2 * half)])[torch.randperm(dim, generator=gen)]
        if i >= 4:
            x[0] += x[0] * (i - 5) * 0.25
        m = float(sum(Fraction(v) for v in x.tolist())) / dim
        rows.append(x)
        want.append((x - torch.tensor(np.float32(m))) * torch.tensor(rstd_of(x, m)))
    look(torch.stack(rows), torch.stack(want), zk.ZK_NORM_LAYER, 16)
