"""What the entry points of quantised inference refuse on the host: nothing here touches a GPU."""
import ctypes

import pytest

P = 1 << 20   # an address that is never read: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def zk():
    import paper_2404_16109_amd as zk
    return zk


def cache(zk, **kw):
    v = dict(k=P, v=P, k_exp=P, v_exp=P, pages=4, kv_heads=2, page_tokens=64, head_dim=128)
    v.update(kw)
    return zk.kvcache_i8(*[v[n] for n, _ in zk.kvcache_i8._fields_])


def seqs(zk, **kw):
    v = dict(cu=P, lens=P, table=P, table_stride=8, table_pages=8, seqs=2, rows=5, max_new=3, max_len=100, fault=None)
    v.update(kw)
    return zk.kv_seqs(*[v[n] for n, _ in zk.kv_seqs._fields_])


def append(zk, c=None, s=None, k=P, v=P, dtype=2):
    c, s = c or cache(zk), s or seqs(zk)
    return zk.raw().kvcache_append(ctypes.byref(c), k, 512, 128, v, 512, 128, dtype, ctypes.byref(s), None)


def attend(zk, c=None, s=None, q=P, out=P, dtype=2, heads=8, scale=0.1, window=0, lse=None, ws=None, ws_bytes=0):
    c, s = c or cache(zk), s or seqs(zk)
    return zk.raw().kvcache_attention(ctypes.byref(c), q, 1024, 128, dtype, heads, ctypes.byref(s), scale, window, out, 1024, 128, lse, ws,
                                      ws_bytes, None)


BAD_CACHES = [dict(k=None), dict(v=None), dict(k_exp=None), dict(v_exp=None), dict(k=P + 8), dict(v=P + 1), dict(pages=0), dict(pages=1 << 31),
              dict(kv_heads=0), dict(kv_heads=20000), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(head_dim=0),
              dict(head_dim=24), dict(head_dim=272)]
BAD_SEQS = [dict(cu=None), dict(lens=None), dict(table=None), dict(cu=P + 2), dict(seqs=65536), dict(rows=1 << 31), dict(max_new=0),
            dict(table_pages=0), dict(table_stride=7), dict(fault=P + 1)]


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches(zk, call, bad):
    assert call(zk, c=cache(zk, **bad)) == zk.ZK_E_BADARG


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad", BAD_SEQS)
def test_sequences(zk, call, bad):
    assert call(zk, s=seqs(zk, **bad)) == zk.ZK_E_BADARG


def test_append_arguments(zk):
    for kw in (dict(k=None), dict(v=None), dict(dtype=3), dict(dtype=4), dict(dtype=-1), dict(k=P + 1), dict(dtype=0, v=P + 2)):
        assert append(zk, **kw) == zk.ZK_E_BADARG, kw
    assert append(zk, s=seqs(zk, rows=0), k=None) == zk.ZK_OK
    assert append(zk, s=seqs(zk, seqs=0), k=None) == zk.ZK_OK


def test_attention_arguments(zk):
    for kw in (dict(q=None), dict(out=None), dict(dtype=0), dict(dtype=3), dict(heads=0), dict(heads=7), dict(heads=131072), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(window=1 << 31), dict(q=P + 1), dict(out=P + 1), dict(lse=P + 2)):
        assert attend(zk, **kw) == zk.ZK_E_BADARG, kw
    assert attend(zk, s=seqs(zk, rows=0), q=None) == zk.ZK_OK
    assert zk.raw().kvcache_attention(None, P, 1, 1, 2, 8, ctypes.byref(seqs(zk)), 0.1, 0, P, 1, 1, None, None, 0, None) == zk.ZK_E_BADARG
    # a long context is shared out: that needs a workspace
    s = seqs(zk, max_len=100000, rows=2, max_new=1)
    need = zk.kvcache_attention_workspace_bytes(2, 2, 1, 8, 2, 128, 100000)
    assert need > 0
    assert attend(zk, s=s) == zk.ZK_E_BUFSZ and attend(zk, s=s, ws=P, ws_bytes=need // 2) == zk.ZK_E_BUFSZ
    assert zk.kvcache_attention_workspace_bytes(0, 2, 1, 8, 2, 128, 100) == 0 and zk.kvcache_attention_workspace_bytes(2, 2, 1, 7, 2, 128, 100) == 0


def test_read_arguments(zk):
    def read(c=None, pages=P, n=5, k=P, v=P):
        return zk.raw().kvcache_read(ctypes.byref(c or cache(zk)), pages, n, k, v, None, None)
    for kw in (dict(pages=None), dict(k=None), dict(v=None), dict(n=1 << 31), dict(k=P + 2), dict(c=cache(zk, head_dim=20))):
        assert read(**kw) == zk.ZK_E_BADARG, kw
    assert read(n=0, pages=None) == zk.ZK_OK


def test_w4_arguments(zk):
    def call(y=P, ys=64, x=P, xs=256, dtype=2, rows=2, codes=P, scales=P, n=64, k=256, group=128):
        return zk.raw().w4_matvec(y, ys, x, xs, dtype, rows, codes, scales, n, k, group, 1.0, None, 0, None)
    for kw in (dict(y=None), dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=4), dict(dtype=-1), dict(n=0), dict(k=0), dict(k=48),
               dict(k=1 << 25), dict(n=1 << 25), dict(group=16), dict(group=256), dict(group=0), dict(codes=P + 8), dict(x=P + 2), dict(xs=255),
               dict(xs=260), dict(ys=63), dict(scales=P + 1), dict(y=P + 1), dict(dtype=3, y=P + 4)):
        assert call(**kw) == zk.ZK_E_BADARG, kw
    assert call(rows=0, x=None, y=None) == zk.ZK_OK
    for kw in (dict(W=None), dict(codes=None), dict(k=33), dict(group=48)):
        a = dict(W=P, codes=P, scales=P, n=8, k=64, group=32)
        a.update(kw)
        assert zk.raw().w4_expand_i16(a["W"], a["codes"], a["scales"], a["n"], a["k"], a["group"], None) == zk.ZK_E_BADARG, kw


def test_logprobs_arguments(zk):
    full = dict(target=P, rank=P, lse=P, entropy=P, top_ids=P, top=P)

    def call(logits=P, stride=1000, dtype=0, rows=2, vocab=1000, targets=P, top=5, out=full, ws=None, ws_bytes=0):
        o = zk.logprobs_out(*[out.get(n) for n, _ in zk.logprobs_out._fields_])
        return zk.raw().logprobs(logits, stride, dtype, rows, vocab, targets, top, ctypes.byref(o), ws, ws_bytes, None)
    for kw in (dict(logits=None), dict(stride=999), dict(dtype=3), dict(dtype=7), dict(vocab=0), dict(vocab=(1 << 19) + 1, stride=1 << 20), dict(top=33),
               dict(top=6, vocab=5), dict(logits=P + 2), dict(out=dict(full, target=None)), dict(out=dict(full, rank=None)),
               dict(out=dict(full, top=None)), dict(out=dict(full, top_ids=None))):
        assert call(**kw) == zk.ZK_E_BADARG, kw
    assert call(rows=0, logits=None) == zk.ZK_OK
    need = zk.logprobs_workspace_bytes(2, 100000, 5)
    assert need > 0 and call(vocab=100000, stride=100000) == zk.ZK_E_BUFSZ
    assert call(vocab=100000, stride=100000, ws=P, ws_bytes=need // 2) == zk.ZK_E_BUFSZ
    assert zk.logprobs_workspace_bytes(0, 1000, 1) == 0 and zk.logprobs_workspace_bytes(5, 1000, 33) == 0
