"""What the entry points of a decoder layer in 8 bits refuse on the host: nothing here touches a GPU."""
import ctypes

import pytest
import torch

from tests.test_serve_binding import Library
from tests.test_serve_binding import OnGpu as OnAGpu
from tests.test_serve_refusals import BAD_CACHES, BAD_SEQS, cache, seqs


class OnGpu(OnAGpu):
    """A host tensor that says on which GPU it is."""

    def __init__(self, *shape, dtype=torch.int32, device=0):
        super().__init__(*shape, dtype=dtype)
        self.device_index = device

    def get_device(self):
        return self.device_index


@pytest.fixture
def stand_in(monkeypatch):
    from paper_2404_16109_amd import binding
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_current", lambda: (0, 0))
    return binding, lib


P = 1 << 20   # an address that is never read: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    return zk


def quantise(zk, codes=P, cs=64, scales=P, x=P, xs=64, dtype=2, rows=2, k=64):
    return zk.raw().i8_quantise(codes, cs, scales, x, xs, dtype, rows, k, None)


def test_quantise(zk):
    for kw in (dict(codes=None), dict(scales=None), dict(x=None), dict(x=P + 1), dict(dtype=0, x=P + 2), dict(scales=P + 2), dict(dtype=3), dict(dtype=4),
               dict(dtype=-1), dict(k=0), dict(k=131057, xs=1 << 18, cs=1 << 18), dict(xs=63), dict(cs=63), dict(rows=1 << 31), dict(xs=1 << 41)):
        assert quantise(zk, **kw) == zk.ZK_E_BADARG, kw
    assert quantise(zk, rows=0, codes=None, x=None, scales=None) == zk.ZK_OK


def matmul(zk, y=P, ys=64, dtype=2, x=P, xs=256, x_scales=P, rows=2, w=P, w_scales=P, n=64, k=256, ws=None, ws_bytes=0):
    return zk.raw().i8_matmul(y, ys, dtype, x, xs, x_scales, rows, w, w_scales, n, k, ws, ws_bytes, None)


def test_matmul(zk):
    for kw in (dict(y=None), dict(x=None), dict(w=None), dict(x_scales=None), dict(w_scales=None), dict(dtype=3), dict(dtype=5), dict(dtype=-1), dict(n=0),
               dict(k=0), dict(k=8), dict(k=24), dict(k=131072, xs=131072), dict(n=(1 << 24) + 1, ys=1 << 25), dict(rows=(1 << 24) + 1), dict(x=P + 8),
               dict(w=P + 8), dict(y=P + 1), dict(dtype=0, y=P + 2), dict(dtype=4, y=P + 2), dict(xs=240), dict(xs=264), dict(xs=(1 << 23) + 16), dict(ys=63),
               dict(x_scales=P + 2), dict(w_scales=P + 1), dict(rows=1 << 24, n=1 << 24, ys=1 << 24)):
        assert matmul(zk, **kw) == zk.ZK_E_BADARG, kw
    assert matmul(zk, rows=0, x=None, y=None, w=None) == zk.ZK_OK
    need = zk.i8_matmul_workspace_bytes(2, 64, 65536)
    assert need > 0
    for dtype in (0, 2, 4):
        assert matmul(zk, k=65536, xs=65536, dtype=dtype) == zk.ZK_E_BUFSZ
        assert matmul(zk, k=65536, xs=65536, dtype=dtype, ws=P, ws_bytes=need // 2) == zk.ZK_E_BUFSZ
    assert zk.i8_matmul_workspace_bytes(0, 64, 65536) == 0 and zk.i8_matmul_workspace_bytes(2, 64, 65537) == 0


def norm(zk, dtype=2, rows=2, dim=64, **kw):
    v = dict(x=P, x_row_stride=64, z=P, z_row_stride=64, gate=P, gate_row_stride=0, post_gain=P, post_bias=P, gain=P, bias=P, r=P, r_row_stride=64, h=P,
             h_row_stride=64, codes=None, codes_row_stride=64, scales=None, post_norm=1, norm=2, alpha=1.0, eps=1e-5)
    v.update(kw)
    a = zk.block_norm_args(*[v[n] for n, _ in zk.block_norm_args._fields_])
    return zk.raw().block_norm(ctypes.byref(a), dtype, rows, dim, None)


def test_norm(zk):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(x=None), dict(dtype=3), dict(dtype=4), dict(dtype=-1), dict(dim=0), dict(dim=65), dict(dim=32769), dict(rows=1 << 31), dict(norm=3),
               dict(norm=-1), dict(post_norm=3), dict(alpha=nan), dict(alpha=inf), dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(z=None),
               dict(z=None, gate=None), dict(z=None, gate=None, post_gain=None, post_bias=None), dict(h=None, r=None), dict(codes=P, scales=P),
               dict(h=None, codes=P), dict(h=None, scales=P), dict(scales=P), dict(x_row_stride=63), dict(z_row_stride=63), dict(r_row_stride=63),
               dict(h_row_stride=63), dict(h=None, codes=P, scales=P, codes_row_stride=63), dict(gate_row_stride=63), dict(x=P + 1), dict(z=P + 1),
               dict(gate=P + 1), dict(r=P + 1), dict(h=P + 1), dict(gain=P + 1), dict(bias=P + 1), dict(post_gain=P + 1), dict(post_bias=P + 1),
               dict(h=None, codes=P, scales=P + 2), dict(dtype=0, x=P + 2)):
        assert norm(zk, **kw) == zk.ZK_E_BADARG, kw
    assert zk.raw().block_norm(None, 2, 2, 64, None) == zk.ZK_E_BADARG
    assert norm(zk, rows=0, x=None, z=None, r=None, h=None) == zk.ZK_OK


def test_sizes_of_the_workspace(zk):
    """Enough outputs, or a k too short to be shared: none."""
    for rows, n, k in ((1, 5120, 5120), (32, 13824, 5120), (8192, 13824, 5120), (1, 16, 1024), (1 << 24, 1, 16)):
        assert zk.i8_matmul_workspace_bytes(rows, n, k) == 0
    for rows, n, k in ((1, 100, 65536), (333, 5120, 13824)):
        assert zk.i8_matmul_workspace_bytes(rows, n, k) >= 2 * 4 * rows * n


def test_python_takes_the_gpus_tensors_only(stand_in):
    zk, lib = stand_in
    i8, f32, bf16 = torch.int8, torch.float32, torch.bfloat16
    x, v = OnGpu(3, 32, dtype=bf16), OnGpu(32, dtype=bf16)
    host = torch.zeros(3, 32, dtype=bf16)
    out = dict(r=OnGpu(3, 32, dtype=bf16), h=OnGpu(3, 32, dtype=i8), scales=OnGpu(3, dtype=f32))
    assert zk.block_norm(x, x, gain=v, gate=v, **out)[0] == 0
    for kw in (dict(z=host), dict(gain=torch.zeros(32, dtype=bf16)), dict(gate=host), dict(r=host), dict(h=torch.zeros(3, 32, dtype=i8)),
               dict(scales=torch.zeros(3)), dict(gain=OnGpu(32, dtype=f32)), dict(z=OnGpu(3, 31, dtype=bf16)), dict(bias=OnGpu(31, dtype=bf16)),
               dict(x=OnGpu(3, 32, dtype=bf16, device=1)), dict(r=OnGpu(3, 32, dtype=bf16, device=1)), dict(gain=OnGpu(32, dtype=bf16, device=1)),
               dict(gate=OnGpu(2, 32, dtype=bf16)), dict(post_gain=OnGpu(33, dtype=bf16)), dict(scales=OnGpu(2, dtype=f32))):
        with pytest.raises(AssertionError):
            zk.block_norm(**dict(dict(x=x, z=x, **out), **kw))
    codes, scales = OnGpu(3, 32, dtype=i8), OnGpu(3, dtype=f32)
    assert zk.i8_quantise(x, codes, scales)[0] == 0
    for a in ((host, codes, scales), (x, torch.zeros(3, 32, dtype=i8), scales), (x, codes, torch.zeros(3)), (x, OnGpu(3, 31, dtype=i8), scales)):
        with pytest.raises(AssertionError):
            zk.i8_quantise(*a)
    w, ws, y = OnGpu(8, 32, dtype=i8), OnGpu(8, dtype=f32), OnGpu(3, 8, dtype=bf16)
    space = OnGpu(4096, dtype=torch.uint8)
    assert zk.i8_matmul(codes, w, scales, ws, out=y, ws=space)[0] == 0
    for kw in (dict(x=torch.zeros(3, 32, dtype=i8)), dict(w=torch.zeros(8, 32, dtype=i8)), dict(x_scales=torch.zeros(3)), dict(w_scales=OnGpu(7, dtype=f32)),
               dict(out=torch.zeros(3, 8, dtype=bf16)), dict(out=OnGpu(3, 9, dtype=bf16)), dict(ws=torch.zeros(4096, dtype=torch.uint8)),
               dict(w=OnGpu(8, 16, dtype=i8)), dict(w=OnGpu(8, 32, dtype=i8, device=1)), dict(ws=OnGpu(4096, dtype=torch.uint8, device=1))):
        with pytest.raises(AssertionError):
            zk.i8_matmul(**dict(dict(x=codes, w=w, x_scales=scales, w_scales=ws, out=y, ws=space), **kw))
    assert set(lib.calls) == {"block_norm", "i8_quantise", "i8_matmul"}


def prefix(zk, c=None, s=None, q=P, out=P, dtype=2, heads=8, scale=0.1, front=P, pages=2, lse=None, ws=None, ws_bytes=0):
    c, s = c or cache(zk), s or seqs(zk)
    return zk.raw().kvcache_attention_prefix(ctypes.byref(c), q, 1024, 128, dtype, heads, ctypes.byref(s), front, pages, scale, out, 1024, 128, lse, ws,
                                             ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_prefix_caches(zk, bad):
    assert prefix(zk, c=cache(zk, **bad)) == zk.ZK_E_BADARG


@pytest.mark.parametrize("bad", BAD_SEQS)
def test_prefix_sequences(zk, bad):
    assert prefix(zk, s=seqs(zk, **bad)) == zk.ZK_E_BADARG


def test_prefix_arguments(zk):
    for kw in (dict(q=None), dict(out=None), dict(dtype=0), dict(dtype=3), dict(dtype=4), dict(heads=0), dict(heads=7), dict(heads=131072),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(q=P + 1), dict(out=P + 1), dict(lse=P + 2), dict(front=None), dict(front=P + 2),
               dict(pages=1 << 25), dict(s=seqs(zk, rows=1 << 24, max_new=1 << 24)), dict(c=cache(zk, kv_heads=1024), heads=1024, s=seqs(zk, seqs=65535, rows=65535, max_new=1)), dict(s=seqs(zk, rows=(1 << 31) - 1, max_new=1))):
        assert prefix(zk, **kw) == zk.ZK_E_BADARG, kw
    assert prefix(zk, s=seqs(zk, rows=0), q=None) == zk.ZK_OK and prefix(zk, s=seqs(zk, seqs=0), q=None) == zk.ZK_OK
    need = zk.kvcache_attention_prefix_workspace_bytes(2, 5, 3, 8, 2, 128, 128, 100)
    assert need > 0 and prefix(zk) == zk.ZK_E_BUFSZ and prefix(zk, ws=P, ws_bytes=need // 2) == zk.ZK_E_BUFSZ
    assert prefix(zk, front=None, pages=0) == zk.ZK_E_BUFSZ   # no prefix: right arguments
    for a in ((0, 5, 3, 8, 2, 128, 128, 100), (2, 0, 3, 8, 2, 128, 128, 100), (2, 5, 0, 8, 2, 128, 128, 100), (2, 5, 3, 7, 2, 128, 128, 100),
              (2, 5, 3, 8, 0, 128, 128, 100), (65536, 5, 3, 8, 2, 128, 128, 100)):
        assert zk.kvcache_attention_prefix_workspace_bytes(*a) == 0


def test_prefix_from_python(stand_in):
    zk, lib = stand_in
    i8, bf16 = torch.int8, torch.bfloat16
    c = zk.KvCache(OnGpu(4, 2, 16, 32, dtype=i8), OnGpu(4, 2, 32, 16, dtype=i8), OnGpu(4, 2, dtype=i8), OnGpu(4, 2, dtype=i8))
    kw = dict(cache=c, q=OnGpu(3, 2, 32, dtype=bf16), cu=OnGpu(2), lens=OnGpu(1), table=OnGpu(1, 4), prefix=OnGpu(2), max_new=3, max_len=60, scale=0.1,
              out=OnGpu(3, 2, 32, dtype=bf16), lse=OnGpu(3, 2, dtype=torch.float32), ws=OnGpu(4096, dtype=torch.uint8))
    assert zk.kvcache_attention_prefix(**kw)[0] == 0
    for bad in (dict(prefix=OnGpu(2, device=1)), dict(q=OnGpu(3, 2, 32, dtype=bf16, device=1)), dict(ws=OnGpu(4096, dtype=torch.uint8, device=1)),
                dict(prefix=torch.zeros(2, dtype=torch.int32)), dict(prefix=OnGpu(2, dtype=torch.int64)), dict(prefix=OnGpu(1, 2)),
                dict(q=torch.zeros(3, 2, 32, dtype=bf16)), dict(out=torch.zeros(3, 2, 32, dtype=bf16)), dict(lse=torch.zeros(3, 2)),
                dict(ws=torch.zeros(4096, dtype=torch.uint8)), dict(fault=torch.zeros(1, dtype=torch.int32)), dict(table=torch.zeros(1, 4, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            zk.kvcache_attention_prefix(**dict(kw, **bad))
    assert lib.calls == ["kvcache_attention_prefix"]


def test_prefix_launches_are_below_2_to_the_32_threads(zk):
    """A wavefront for each row of a sequence and head, four to a workgroup: the largest call that fits wants its workspace, the next is
    refused before anything is enqueued."""
    c = cache(zk, kv_heads=1)
    for rows, want in (((1 << 26) - 4, zk.ZK_E_BUFSZ), ((1 << 26) - 3, zk.ZK_E_BADARG), ((1 << 26) - 2, zk.ZK_E_BADARG), ((1 << 26) - 1, zk.ZK_E_BADARG)):
        assert prefix(zk, c=c, heads=1, s=seqs(zk, seqs=1, rows=rows, max_new=rows)) == want, rows
    for rows, want in (((1 << 21) - 1, zk.ZK_E_BUFSZ), (1 << 21, zk.ZK_E_BADARG)):   # 32 heads
        assert prefix(zk, c=c, heads=32, s=seqs(zk, seqs=1, rows=rows, max_new=rows)) == want, rows


@pytest.mark.parametrize("seqs_,rows,max_new,prefix_tokens,max_len", [
    (128, 2048 + 127, 2048, 8192, 10240), (256, 4096 + 255, 4096, 2048, 8000), (64, 64, 1, 8192, 8704), (16, 490, 64, 32768, 33068), (1, 5000, 5000, 4096, 5000),
    (65535, 65535, 1, 512, 600), (700, 700 + 299, 300, 0, 900)])
def test_workspace_of_a_prefix_goes_by_rows(zk, seqs_, rows, max_new, prefix_tokens, max_len):
    """A prompt's next part beside single tokens wants no more than its rows do: 32 parts of the prefix and 32 own ones at most, and some where
    either has one tile only."""
    for heads, kv, d in ((40, 8, 128), (16, 16, 64), (8, 1, 256)):
        need = zk.kvcache_attention_prefix_workspace_bytes(seqs_, rows, max_new, heads, kv, d, prefix_tokens, max_len)
        part = rows * heads * 4 * (d + 2)
        own = max(max_len - prefix_tokens, 1)
        most = min(32, -(-prefix_tokens // 64)) + min(32, -(-own // 256))   # own parts have four tiles at least
        assert part <= need <= part * most + 4096, (need, part)
    # beside many sequences nothing of their own is shared out: parts of the prefix and one more
    if seqs_ == 128:
        assert zk.kvcache_attention_prefix_workspace_bytes(seqs_, rows, max_new, 40, 8, 128, prefix_tokens, max_len) < 1 << 30
