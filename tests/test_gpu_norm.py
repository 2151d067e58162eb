"""block_norm and i8_quantise against their definition, bit for bit, and against the formula in 64 bits."""
import itertools
import math

import pytest
import torch

import paper_2404_16109_amd as zk
from tests import layer_ref as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


def tensor(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def on_gpu(kw):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}


def same(a, b):
    """Bit for bit, any NaN like another."""
    a, b = a.cpu(), b.cpu()
    assert a.dtype == b.dtype and a.shape == b.shape
    nan = torch.isnan(a.double()) & torch.isnan(b.double())
    bad = ~((a == b) | nan)
    assert not bad.any(), (int(bad.sum()), a[bad][:4], b[bad][:4])


def case(rows, dim, dtype, norm, post, gate, biased, block=True, seed=0, mean=0.0):
    gen = torch.Generator().manual_seed(rows * 1000003 + dim * 101 + seed)
    kw = {"norm": norm, "gain": tensor(gen, dim, dtype=dtype) + 1, "eps": 1e-5}
    x = tensor(gen, rows, dim, dtype=dtype, scale=2.0) + mean
    if biased:
        kw["bias"] = tensor(gen, dim, dtype=dtype)
    z = None
    if block:
        z = tensor(gen, rows, dim, dtype=dtype) * 3
        kw["post_norm"], kw["alpha"] = post, 0.7
        if post:
            kw["post_gain"] = tensor(gen, dim, dtype=dtype)
            if biased:
                kw["post_bias"] = tensor(gen, dim, dtype=dtype)
        if gate:
            kw["gate"] = tensor(gen, dim, dtype=dtype) if gate == 1 else tensor(gen, rows, dim, dtype=dtype)
    return x, z, kw


def check(x, z, kw, quantise):
    want_r, want_h = ref.norm_steps(x, z, **kw)
    rc, r, h, scales = zk.block_norm(x.cuda(), None if z is None else z.cuda(), quantise=quantise, **on_gpu(kw))
    assert rc == zk.ZK_OK
    same(r, want_r)
    if quantise:
        codes, want = ref.codes_of(want_h)
        same(scales, want)
        same(h, codes)
        return
    same(h, want_h.to(x.dtype))
    # each step of the norm, its statistics and its store are off by half a step of their type at most
    h64, size = ref.norm_formula(want_r, kw["norm"], kw.get("gain"), kw.get("bias"), kw["eps"])
    least = 2.0 ** -149 if x.dtype != F16 else 2.0 ** -25
    none = torch.isnan(h64)   # of rows that are not finite; those are held to the definition above
    assert (none == torch.isnan(h.cpu())).all()
    assert (none | ((h.cpu().double() - h64).abs() <= HALF[x.dtype] * h64.abs() + 8 * 2.0 ** -24 * size + least)).all()


# widths: one element, odd ones, runs that end inside a thread's, every number of elements to a thread, the widest
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 63, 64, 65, 520, 1023, 4096, 4097, 5120, 8200, 16384, 16392, 32767, 32768])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_widths(dim, dtype):
    for norm, quantise in itertools.product((zk.ZK_NORM_RMS, zk.ZK_NORM_LAYER), (False, True)):
        check(*case(3, dim, dtype, norm, zk.ZK_NORM_NONE, 1, norm == zk.ZK_NORM_LAYER), quantise)


@pytest.mark.parametrize("dim", [1024, 1032, 5120, 8192, 16384])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_many_rows(dim, dtype):
    for norm, quantise in ((zk.ZK_NORM_RMS, True), (zk.ZK_NORM_LAYER, False)):
        check(*case(1024, dim, dtype, norm, zk.ZK_NORM_RMS, 1, False), quantise)


@pytest.mark.parametrize("dim", [8193, 16385, 20000, 32768])
def test_long_rows_of_all_kinds(dim):
    for i, (norm, post, gate, biased) in enumerate(itertools.product((0, 1, 2), (0, 1, 2), (0, 1, 2), (False, True))):
        if i % 4 == dim % 4:
            check(*case(2, dim, (F32, F16, BF16)[i % 3], norm, post, gate, biased), bool(i & 2))
    check(*case(3, dim, BF16, zk.ZK_NORM_RMS, 0, 0, False, block=False), True)


@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("gate", [0, 1, 2])
@pytest.mark.parametrize("biased", [False, True])
def test_all_kinds(norm, post, gate, biased):
    for dtype, dim, quantise in ((F32, 260, False), (F32, 261, True), (F16, 264, True), (BF16, 264, False), (BF16, 133, True)):
        check(*case(5, dim, dtype, norm, post, gate, biased), quantise)


@pytest.mark.parametrize("rows", [1, 2, 255, 1000])
def test_rows_without_a_block(rows):
    for quantise in (False, True):
        check(*case(rows, 640, BF16, zk.ZK_NORM_RMS, 0, 0, False, block=False), quantise)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_mean_far_from_zero(dtype):
    """A variance that would drown in 32 bits beside the square of the mean."""
    for quantise in (False, True):
        check(*case(4, 1000, dtype, zk.ZK_NORM_LAYER, 0, 0, True, block=False, mean=1000.0), quantise)


def test_numbers_at_the_ends():
    """Zeros, subnormals, the largest and smallest, infinities and NaN, each in a row of its own; neighbours are as without."""
    x, z, kw = case(12, 256, F32, zk.ZK_NORM_RMS, 0, 0, True, block=False)
    x[1] = 0.0
    x[2] *= 1e-42
    x[3] *= 1e30
    x[4, 7] = math.inf
    x[5, 255] = math.nan
    x[6] = 3.4e38
    x[7] = 0.0
    x[7, 3] = -1e-38
    x[8, 0] = -math.inf
    for quantise in (False, True):
        check(x, z, kw, quantise)
    for norm in (zk.ZK_NORM_NONE, zk.ZK_NORM_LAYER):
        kw["norm"] = norm
        kw.pop("bias", None)
        check(x, z, kw, True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("k", [1, 5, 8, 128, 777, 4096, 13824, 32768, 32769, 50000])
def test_quantise(dtype, k):
    gen = torch.Generator().manual_seed(k)
    x = tensor(gen, 4, k, dtype=dtype, scale=3.0)
    x[1] = 0.0
    x[2, k // 2] = math.nan if k % 2 else math.inf
    rc, codes, scales = zk.i8_quantise(x.cuda())
    assert rc == zk.ZK_OK
    want = ref.codes_of(x.float())
    same(codes, want[0])
    same(scales, want[1])
    assert codes[0].abs().max() == 127 and scales[1] == 0 and torch.isnan(scales[2]) and not codes[2].any()


def test_quantise_borders():
    """Values in the middle between two codes go to the even one."""
    x = torch.arange(-127, 128, dtype=F32)[None].repeat(3, 1)
    x[1, 1:-1] += 0.5
    x[2, 1:-1] -= 0.5
    rc, codes, scales = zk.i8_quantise(x.cuda())
    assert rc == zk.ZK_OK and (scales == 1).all()
    same(codes, torch.round(x).to(torch.int8))


def test_quantise_next_to_nothing():
    x = torch.zeros(4, 64)
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = 2.0 ** -100, 2.0 ** -101, 1e-45, 3.4e38
    rc, codes, scales = zk.i8_quantise(x.cuda())
    assert rc == zk.ZK_OK
    same(codes, ref.codes_of(x)[0])
    same(scales, ref.codes_of(x)[1])
    assert codes[:, 0].tolist() == [127, 0, 0, 127]


def strided(t, pad, offset):
    """The same values in a wider tensor, beginning `offset` elements in; what lies around is poison."""
    rows, cols = t.shape
    whole = torch.full((rows * (cols + pad) + offset + 64,), 77, dtype=t.dtype, device="cuda")
    view = whole[offset:offset + rows * (cols + pad)].reshape(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view, whole


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (8, 8), (1, 0), (3, 5), (16, 1)])
@pytest.mark.parametrize("quantise", [False, True])
def test_strides(dtype, pad, offset, quantise):
    x, z, kw = case(6, 264, dtype, zk.ZK_NORM_LAYER, zk.ZK_NORM_RMS, 2, True)
    kw_g = on_gpu(kw)
    (xs, _), (zs, _), (kw_g["gate"], _) = (strided(t, pad, offset) for t in (x, z, kw["gate"]))
    r, r_all = strided(torch.zeros(6, 264, dtype=dtype), pad, offset)
    h, h_all = strided(torch.zeros(6, 264, dtype=torch.int8 if quantise else dtype), pad, offset)
    rc, r2, h2, scales = zk.block_norm(xs, zs, r=r, h=h, **kw_g)
    assert rc == zk.ZK_OK
    want_r, want_h = ref.norm_steps(x, z, **kw)
    same(r2, want_r)
    same(h2, ref.codes_of(want_h)[0] if quantise else want_h.to(dtype))
    for whole in (r_all, h_all):   # nothing around them is written
        assert int((whole == 77).sum()) >= whole.numel() - 6 * 264
        body = whole[offset:offset + 6 * (264 + pad)].reshape(6, 264 + pad)[:, 264:]
        assert (body == 77).all() and (whole[:offset] == 77).all() and (whole[offset + 6 * (264 + pad):] == 77).all()


@pytest.mark.parametrize("dim", [264, 261])
def test_in_place_either_way_round(dim):
    for swap in (False, True):
        x, z, kw = case(9, dim, BF16, zk.ZK_NORM_RMS, zk.ZK_NORM_RMS, 1, False)
        want_r, want_h = ref.norm_steps(x, z, **kw)
        xg, zg = x.cuda(), z.cuda()
        rc, r, h, _ = zk.block_norm(xg, zg, r=zg if swap else xg, h=xg if swap else zg, **on_gpu(kw))
        assert rc == zk.ZK_OK
        same(r, want_r)
        same(h, want_h.to(BF16))


def test_r_alone():
    """Behind the last block there is nothing to norm; r in place."""
    x, z, _ = case(4, 100, F16, 0, 0, 0, False)
    a = zk.block_norm_args()
    xg, zg = x.cuda(), z.cuda()
    a.x, a.x_row_stride, a.z, a.z_row_stride, a.r, a.r_row_stride, a.alpha = xg.data_ptr(), 100, zg.data_ptr(), 100, xg.data_ptr(), 100, 1.0
    import ctypes
    assert zk.raw().block_norm(ctypes.byref(a), zk.ZK_F16, 4, 100, torch.cuda.current_stream().cuda_stream) == zk.ZK_OK
    same(xg, (x.float() + z.float()).to(F16))


def test_gate_of_all_tokens_by_stride():
    x, z, kw = case(5, 64, F32, zk.ZK_NORM_RMS, 0, 1, False)
    one = zk.block_norm(x.cuda(), z.cuda(), **on_gpu(kw))
    kw["gate"] = kw["gate"][None].expand(5, 64)
    many = zk.block_norm(x.cuda(), z.cuda(), **on_gpu(dict(kw, gate=kw["gate"].contiguous())))
    same(one[1], many[1])
    same(one[2], many[2])


def test_no_rows():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    rc, r, h, scales = zk.block_norm(x, x, gate=torch.zeros(64, dtype=BF16, device="cuda"), quantise=True)
    assert rc == zk.ZK_OK and h.shape == (0, 64) and scales.shape == (0,)
    assert zk.i8_quantise(x)[0] == zk.ZK_OK


def test_many_short_rows():
    x, z, kw = case(70001, 16, BF16, zk.ZK_NORM_RMS, 0, 1, False)
    check(x, z, kw, True)


def test_more_rows_than_a_launch_has_threads_for():
    """Rows times the threads of each are more than 2^32."""
    rows = (1 << 26) + 1234567
    x = torch.zeros(rows, 1, dtype=F16, device="cuda")
    x[::3] = -2.0
    x[-1] = 5.0
    rc, codes, scales = zk.i8_quantise(x)
    assert rc == zk.ZK_OK
    assert (codes[::3][:-1] == -127).all() and codes[-1] == 127 and not codes[1::3][:-1].any() and not codes[2::3][:-1].any()
    step = torch.tensor(2.0, dtype=F32) / torch.tensor(127.0, dtype=F32)
    assert (scales[::3][:-1] == step.item()).all() and scales[-1] == (torch.tensor(5.0) / torch.tensor(127.0)).item()
    rc, r, h, _ = zk.block_norm(x, x, norm=zk.ZK_NORM_NONE)
    assert rc == zk.ZK_OK and torch.equal(r, x + x) and torch.equal(h, r)


def test_other_stream_and_graph():
    x, z, kw = case(40, 520, BF16, zk.ZK_NORM_RMS, zk.ZK_NORM_LAYER, 2, True)
    xg, zg, kwg = x.cuda(), z.cuda(), on_gpu(kw)
    h, scales, r = torch.empty(40, 520, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda"), torch.empty_like(xg)
    codes2, scales2 = torch.empty_like(h), torch.empty_like(scales)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def both():
        assert zk.block_norm(xg, zg, r=r, h=h, scales=scales, **kwg)[0] == zk.ZK_OK
        assert zk.i8_quantise(r, codes2, scales2)[0] == zk.ZK_OK

    with torch.cuda.stream(stream):
        both()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(4):
        x, z, _ = case(40, 520, BF16, zk.ZK_NORM_RMS, zk.ZK_NORM_LAYER, 2, True, seed=seed)
        xg.copy_(x)
        zg.copy_(z)
        graph.replay()
        want_r, want_h = ref.norm_steps(x, z, **kw)
        same(r, want_r)
        same(h, ref.codes_of(want_h)[0])
        same(codes2, ref.codes_of(want_r.float())[0])
