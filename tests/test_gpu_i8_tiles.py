"""i8_matmul on every way it has through its kernels (held to the plan by test_i8_plan.py), bit for bit: whole and with odd ends, with strides."""
import pytest
import torch

import paper_2404_16109_amd as zk
from tests import layer_ref as ref
from tests.i8_sizes import ALL, WAYS, name
from tests.test_gpu_i8 import check, inputs
from tests.test_gpu_norm import same

pytestmark = pytest.mark.gpu

F32, F16, BF16, I32 = torch.float32, torch.float16, torch.bfloat16, torch.int32


@pytest.mark.parametrize("way,size", ALL, ids=lambda x: name(x) if isinstance(x[0], str) else "%d-%d-%d" % x)
def test_ways(way, size):
    assert (zk.i8_matmul_workspace_bytes(*size) > 0) == way[3]
    for dtype in (I32, F32, F16, BF16):
        check(*size, dtype)


@pytest.mark.parametrize("way", WAYS, ids=name)
@pytest.mark.parametrize("dtype", [I32, F32, BF16])
def test_strides(way, dtype):
    """x in a wider tensor whose rest is not zero, y at odd strides and addresses, what lies around it and behind the workspace left as it was."""
    rows, n, k = WAYS[way][0]
    x, w, xs, ws = inputs(rows, n, k)
    wide = torch.full((rows, k + 48), 55, dtype=torch.int8, device="cuda")
    wide[:, 16:16 + k] = x
    want = ref.product(x, w, xs, ws, dtype)
    need = zk.i8_matmul_workspace_bytes(rows, n, k)
    space = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    for pad, offset in ((5, 0), (1, 1), (8 - n % 8, 8)):
        whole = torch.full((rows * (n + pad) + offset + 8,), 77, dtype=dtype, device="cuda")
        y = whole[offset:offset + rows * (n + pad)].reshape(rows, n + pad)[:, :n]
        rc, _ = zk.i8_matmul(wide[:, 16:16 + k], w, xs, ws, out=y, ws=space[:need] if need else None)
        assert rc == zk.ZK_OK
        same(y, want)
        rest = whole[offset:offset + rows * (n + pad)].reshape(rows, n + pad)[:, n:]
        assert (rest == 77).all() and (whole[:offset] == 77).all() and (whole[offset + rows * (n + pad):] == 77).all()
        assert space[need:].eq(0xff).all()


@pytest.mark.parametrize("way", [w for w in WAYS if w[3]], ids=name)
def test_largest_sums_in_parts(way):
    """-128 * -128 over all of k, on every way that adds parts up."""
    rows, n, k = WAYS[way][0]
    x = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    w[n // 2] = 127
    rc, y = zk.i8_matmul(x, w, dtype=I32)
    assert rc == zk.ZK_OK
    want = torch.full((rows, n), 128 * 128 * k, dtype=torch.int32)
    want[:, n // 2] = -128 * 127 * k
    same(y, want)
