"""i8_matmul against the sums in 64 bits, bit for bit."""
import pytest
import torch

import paper_2404_16109_amd as zk
from tests import layer_ref as ref
from tests.test_gpu_norm import same

pytestmark = pytest.mark.gpu

F32, F16, BF16, I32 = torch.float32, torch.float16, torch.bfloat16, torch.int32


def inputs(rows, n, k, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + n * 11 + k + seed)
    x = torch.randint(-128, 128, (rows, k), generator=gen, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=gen, device="cuda", dtype=torch.int8)
    return x, w, torch.rand(rows, generator=gen, device="cuda") + 0.01, torch.rand(n, generator=gen, device="cuda") * 1e-3


def check(rows, n, k, dtype=I32, seed=0):
    x, w, xs, ws = inputs(rows, n, k, seed)
    rc, y = zk.i8_matmul(x, w, xs, ws, dtype=dtype)
    assert rc == zk.ZK_OK
    same(y, ref.product(x, w, xs, ws, dtype))


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 129, 300])
@pytest.mark.parametrize("n", [1, 3, 16, 31, 130, 513])
def test_sizes(rows, n):
    for k in (16, 48, 128, 144, 272, 1040):
        check(rows, n, k)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows", [1, 20, 50, 70, 200])
def test_types(dtype, rows):
    for n, k in ((64, 256), (67, 400), (514, 1024)):
        check(rows, n, k, dtype)


@pytest.mark.parametrize("rows,n,k", [(1, 96, 20000), (5, 40, 131056), (64, 17, 9008), (65, 100, 6416), (333, 300, 4112), (100, 1000, 27200)])
def test_shared_k(rows, n, k):
    """Few outputs and a long k: workgroups share it, and a launch joins them."""
    assert zk.i8_matmul_workspace_bytes(rows, n, k) > 0
    for dtype in (I32, BF16):
        check(rows, n, k, dtype)


@pytest.mark.parametrize("rows,n,k", [(3000, 4200, 272), (4097, 3333, 144), (256, 49152, 128), (49152, 256, 400), (60000, 255, 16), (2048, 6400, 1040)])
def test_large(rows, n, k):
    assert zk.i8_matmul_workspace_bytes(rows, n, k) == 0
    check(rows, n, k)
    check(rows, n, k, F16)


@pytest.mark.parametrize("rows,n,k", [(16, 12801, 400), (32, 12805, 272), (5, 4100, 272), (31, 4099, 144), (20, 2100, 8208), (2000, 5100, 528), (380, 32000, 144),
                                      (190, 12900, 1040), (1537, 8193, 272)])
def test_every_tile(rows, n, k):
    """16 to 64 outputs to a workgroup of few rows, tiles of 128 x 128, 256 x 192 and 256 x 256, all with odd ends."""
    for dtype in (I32, F32, BF16):
        check(rows, n, k, dtype)


@pytest.mark.parametrize("rows,n", [(1, 33), (40, 20), (200, 130)])
def test_largest_sums(rows, n):
    """-128 * -128 over the longest k: 2147221504, just below 2^31; and its negative."""
    k = zk.I8_MAX_K
    x = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[n // 2] = 127
    rc, y = zk.i8_matmul(x, w, dtype=I32)
    assert rc == zk.ZK_OK
    want = torch.full((rows, n), 128 * 128 * k, dtype=torch.int32)
    want[:, n // 2] = -128 * 127 * k
    same(y, want)


@pytest.mark.parametrize("rows", [1, 10, 40, 100, 700])
@pytest.mark.parametrize("dtype", [I32, F32, BF16])
def test_strides(rows, dtype):
    """x in a wider tensor whose rest is not zero; y with odd strides and addresses; nothing beside it is written."""
    n, k = 131, 272
    x, w, xs, ws = inputs(rows, n, k)
    wide = torch.full((rows, k + 48), 55, dtype=torch.int8, device="cuda")
    wide[:, 16:16 + k] = x
    for pad, offset in ((0, 0), (5, 0), (1, 1), (4, 8)):
        whole = torch.full((rows * (n + pad) + offset + 8,), 77, dtype=dtype, device="cuda")
        y = whole[offset:offset + rows * (n + pad)].reshape(rows, n + pad)[:, :n]
        rc, _ = zk.i8_matmul(wide[:, 16:16 + k], w, xs, ws, out=y)
        assert rc == zk.ZK_OK
        same(y, ref.product(x, w, xs, ws, dtype))
        rest = whole[offset:offset + rows * (n + pad)].reshape(rows, n + pad)[:, n:]
        assert (rest == 77).all() and (whole[:offset] == 77).all() and (whole[offset + rows * (n + pad):] == 77).all()


@pytest.mark.parametrize("rows", [1, 100])
def test_scale_that_is_none(rows):
    x, w, xs, ws = inputs(rows, 50, 128)
    xs[0] = float("nan")
    ws[7] = float("inf")
    rc, y = zk.i8_matmul(x, w, xs, ws, dtype=F32)
    assert rc == zk.ZK_OK and torch.isnan(y[0]).all()
    same(y, ref.product(x, w, xs, ws, F32))


def test_workspace_is_needed_and_shared():
    x, w, xs, ws = inputs(5, 40, 40000)
    need = zk.i8_matmul_workspace_bytes(5, 40, 40000)
    small = torch.empty(need // 2, dtype=torch.uint8, device="cuda")
    assert zk.i8_matmul(x, w, xs, ws, ws=small)[0] == zk.ZK_E_BUFSZ
    space = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")
    for offset in (0, 1, 16):   # any address, and what was left there does not matter
        rc, y = zk.i8_matmul(x, w, xs, ws, ws=space[offset:offset + need])
        assert rc == zk.ZK_OK
        same(y, ref.product(x, w, xs, ws, BF16))


def test_no_rows():
    x = torch.empty(0, 64, dtype=torch.int8, device="cuda")
    w = torch.zeros(8, 64, dtype=torch.int8, device="cuda")
    rc, y = zk.i8_matmul(x, w, dtype=I32)
    assert rc == zk.ZK_OK and y.shape == (0, 8)


def test_other_stream_and_graphs_that_share_a_workspace():
    shapes = ((1, 100, 20000), (100, 130, 8000), (300, 513, 528))
    space = torch.empty(max(zk.i8_matmul_workspace_bytes(*s) for s in shapes), dtype=torch.uint8, device="cuda")
    made = []
    for s in shapes:
        x, w, xs, ws = inputs(*s)
        y = torch.empty(s[0], s[1], dtype=BF16, device="cuda")
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            assert zk.i8_matmul(x, w, xs, ws, out=y, ws=space)[0] == zk.ZK_OK
        stream.synchronize()
        same(y, ref.product(x, w, xs, ws, BF16))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert zk.i8_matmul(x, w, xs, ws, out=y, ws=space)[0] == zk.ZK_OK
        made.append((graph, s, x, w, xs, ws, y))
    for seed in range(1, 4):
        for graph, s, x, w, xs, ws, y in made:
            for old, new in zip((x, w, xs, ws), inputs(*s, seed=seed)):
                old.copy_(new)
            graph.replay()
        for _, s, x, w, xs, ws, y in made:
            same(y, ref.product(x, w, xs, ws, BF16))


def test_codes_of_rows_through_a_product():
    """What i8_quantise makes, i8_matmul takes: the result is x w within what 8 bits hold, and a row that is not finite is NaN."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(20, 512, generator=gen, device="cuda")
    x[3, 9] = float("inf")
    w = torch.randn(96, 512, generator=gen, device="cuda")
    _, cx, sx = zk.i8_quantise(x)
    _, cw, sw = zk.i8_quantise(w)
    rc, y = zk.i8_matmul(cx, cw, sx, sw, dtype=F32)
    assert rc == zk.ZK_OK and torch.isnan(y[3]).all()
    keep = [i for i in range(20) if i != 3]
    x64, w64 = x[keep].double(), w.double()
    # a code is off by half a scale (and the roundings of 127 / amax and of the product), on either side of the product
    hx, hw = 0.5001 * sx[keep].double()[:, None], 0.5001 * sw.double()[None]
    bound = hx * w64.abs().sum(1)[None] + hw * x64.abs().sum(1)[:, None] + 512 * hx * hw
    assert ((y[keep].double() - x64 @ w64.t().contiguous()).abs() <= bound * 1.001 + 1e-5).all()
