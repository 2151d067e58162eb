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
