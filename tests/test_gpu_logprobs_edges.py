"""Log probabilities of logits that lie far from zero: what all logits of a row have in common takes nothing from them.

Tolerance: logits are whole numbers, so differences to the largest are exact; the sum and its logarithm are off by 64 * 2^-24
* (1 + entropy) as in test_gpu_logprobs, and the last subtraction rounds to 2^-24 of its result, twice for good measure."""
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


@pytest.mark.parametrize("shift", [0, 40, 20000, -20000, 1 << 22, -(1 << 22)])
@pytest.mark.parametrize("rows,vocab", [(3, 1000), (2, 20011), (2, 70001), (200, 9001)])
def test_what_logits_have_in_common(zk, rows, vocab, shift):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn(rows, vocab, generator=gen, device="cuda") * 4).round()
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    want = serve_ref.logprobs(x[:3], targets[:3].tolist(), 6)
    rc, got = zk.logprobs(x + shift, targets, 6)
    assert rc == zk.ZK_OK
    for r in range(min(rows, 3)):
        tol = 64 * STEP * (1 + want["entropy"][r])
        assert got["top_ids"][r].tolist() == want["top_ids"][r] and got["rank"][r].item() == want["rank"][r]
        for a, b in zip([got["target"][r].item()] + got["top"][r].tolist(), [want["target"][r]] + want["top"][r]):
            assert abs(a - b) <= tol + 2 * STEP * abs(b), (r, a, b)
        assert abs(got["entropy"][r].item() - want["entropy"][r]) <= tol * (1 + want["entropy"][r])
