"""What the Python entry points of quantised inference refuse before the library sees it: addresses that are not the GPU's.
Tensors here are the host's and only say that they are on a GPU; the library is a stand-in that counts calls."""
import ctypes

import pytest
import torch

P = 1 << 20   # an address that is never read


class OnGpu:
    """A host tensor that says it is on the GPU."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.int32):
        self.t = torch.zeros(shape, dtype=dtype)

    def __getattr__(self, name):
        return getattr(self.t, name)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *a: 4096
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def stand_in(monkeypatch):
    from paper_2404_16109_amd import binding
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    return binding, lib


def calls(zk):
    """Each entry point, to be called with fault or ws."""
    i8, bf16 = torch.int8, torch.bfloat16
    cache = zk.KvCache(OnGpu(4, 2, 16, 32, dtype=i8), OnGpu(4, 2, 32, 16, dtype=i8), OnGpu(4, 2, dtype=i8), OnGpu(4, 2, dtype=i8))
    x, seqs = OnGpu(3, 2, 32, dtype=bf16), (OnGpu(2), OnGpu(1), OnGpu(1, 4))
    out = {"out": OnGpu(3, 2, 32, dtype=bf16), "lse": OnGpu(3, 2, dtype=torch.float32)}
    return {
        "append": lambda **kw: zk.kvcache_append(cache, x, x, *seqs, 3, **kw),
        "attend": lambda **kw: zk.kvcache_attention(cache, x, *seqs, 3, 3, 0.1, **dict({"ws": OnGpu(4096, dtype=torch.uint8)}, **kw), **out),
        "read": lambda **kw: zk.kvcache_read(cache, OnGpu(4), 5, **kw),
        "product": lambda **kw: zk.w4_matvec(OnGpu(3, 64, dtype=bf16), OnGpu(8, 32, dtype=torch.uint8), OnGpu(8, 2, dtype=torch.int16), 32,
                                             out=OnGpu(3, 8, dtype=bf16), **kw),
        "logprobs": lambda **kw: zk.logprobs(OnGpu(3, 100, dtype=bf16), None, 2, **kw),
    }


@pytest.mark.parametrize("name", ["append", "attend", "read"])
def test_faults(stand_in, name):
    zk, lib = stand_in
    call = calls(zk)[name]
    for bad in (torch.zeros(1, dtype=torch.int32), OnGpu(1, dtype=torch.int64), OnGpu(1, dtype=torch.uint8), OnGpu(0), OnGpu(2)):
        with pytest.raises(AssertionError, match="fault"):
            call(fault=bad)
    assert lib.calls == []
    call(fault=None)
    call(fault=OnGpu(1))
    assert len(lib.calls) == 2


@pytest.mark.parametrize("name", ["attend", "product", "logprobs"])
def test_workspaces(stand_in, name):
    zk, lib = stand_in
    call = calls(zk)[name]
    strided = OnGpu(4096, dtype=torch.uint8)
    strided.t = torch.zeros(1, dtype=torch.uint8).expand(4096)
    for bad in (torch.zeros(4096, dtype=torch.uint8), strided):
        with pytest.raises(AssertionError, match="ws"):
            call(ws=bad)
    assert lib.calls == []
    call(ws=OnGpu(4096, dtype=torch.uint8))
    assert len(lib.calls) == 1


def test_the_library_refuses_a_fault_word_that_is_not_aligned():
    import paper_2404_16109_amd as zk
    cache = zk.kvcache_i8(P, P, P, P, 4, 2, 64, 128)
    assert zk.raw().kvcache_read(ctypes.byref(cache), P, 5, P, P, P + 2, None) == zk.ZK_E_BADARG
