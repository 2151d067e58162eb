"""A decoder layer in 8 bits, for a batch behind a prompt that it shares: every step against its definition on what it was given, the
whole in a captured graph, and the proof of one of its products."""
import pytest
import torch

import paper_2404_16109_amd as zk
from tests import layer_ref as ref
from tests.test_gpu_norm import same
from tests.test_gpu_prefix import check as check_attention

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DIM, HEADS, KV, HEAD, INNER, T = 256, 8, 2, 32, 512, 16


def weights(gen, n, k):
    """Codes and scales of an n x k matrix, made by the operator that makes those of activations."""
    rc, codes, scales = zk.i8_quantise(torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5)
    assert rc == zk.ZK_OK
    return codes, scales


class Layer:
    def __init__(self, seed, shared, own):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gen, seqs = gen, len(own)
        pages = -(-(shared + max(own)) // T)
        self.prefix = torch.arange(shared // T, dtype=torch.int32, device="cuda")
        mine = torch.arange(seqs * pages, dtype=torch.int32, device="cuda").view(seqs, pages) + shared // T
        self.table = torch.cat([self.prefix[None].expand(seqs, -1), mine], 1)[:, :pages + shared // T].contiguous()
        self.table[:, :shared // T] = -1    # the prefix has pages of its own
        self.cache = zk.KvCache.empty(int(mine.max()) + 1, KV, T, HEAD)
        self.lens = torch.tensor([shared + n for n in own], dtype=torch.int32, device="cuda")
        self.cu = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
        self.most, self.shared = shared + max(own), shared
        self.fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        # the prompt, then each sequence's own tokens, are in the cache
        self.fill([0, shared], [shared], [self.prefix.tolist()])
        for b, n in enumerate(own):
            if n > 1:
                self.fill([0, n - 1], [shared + n - 1], [self.table[b].tolist()])
        self.gains = [(1 + 0.2 * torch.randn(DIM, generator=gen, device="cuda")).to(BF16) for _ in range(3)]
        self.gate = torch.rand(DIM, generator=gen, device="cuda").to(BF16)
        self.qkv, self.out = weights(gen, (HEADS + 2 * KV) * HEAD, DIM), weights(gen, DIM, HEADS * HEAD)
        self.up, self.down = weights(gen, INNER, DIM), weights(gen, DIM, INNER)

    def fill(self, cu, lens, table):
        k, v = (torch.randn(cu[-1], KV, HEAD, generator=self.gen, device="cuda").to(BF16) for _ in range(2))
        cu, lens, table = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (cu, lens, table))
        assert zk.kvcache_append(self.cache, k, v, cu, lens, table, k.shape[0], fault=self.fault) == zk.ZK_OK

    def forward(self, x):
        """Everything that the steps give, in order."""
        s = {"x": x}

        def ok(rc, *got):
            assert rc == zk.ZK_OK
            return got

        s["r0"], s["h0"], s["s0"] = ok(*zk.block_norm(x, gain=self.gains[0], quantise=True))
        s["qkv"], = ok(*zk.i8_matmul(s["h0"], self.qkv[0], s["s0"], self.qkv[1]))
        q, k, v = s["qkv"].view(-1, HEADS + 2 * KV, HEAD).split([HEADS, KV, KV], 1)
        s["q"] = q
        ok(zk.kvcache_append(self.cache, k, v, self.cu, self.lens, self.table, 1, fault=self.fault))
        s["a"], s["lse"] = ok(*zk.kvcache_attention_prefix(self.cache, q, self.cu, self.lens, self.table, self.prefix, 1, self.most, HEAD ** -0.5,
                                                           fault=self.fault))
        flat = s["a"].view(-1, HEADS * HEAD)
        s["ca"], s["sa"] = ok(*zk.i8_quantise(flat))
        s["o"], = ok(*zk.i8_matmul(s["ca"], self.out[0], s["sa"], self.out[1]))
        s["r1"], s["h1"], s["s1"] = ok(*zk.block_norm(x, s["o"], gain=self.gains[1], post_norm=zk.ZK_NORM_RMS, post_gain=self.gains[2], gate=self.gate, quantise=True))
        s["u"], = ok(*zk.i8_matmul(s["h1"], self.up[0], s["s1"], self.up[1], dtype=F32))
        s["cu"], s["su"] = ok(*zk.i8_quantise(torch.relu(s["u"])))
        s["d"], = ok(*zk.i8_matmul(s["cu"], self.down[0], s["su"], self.down[1]))
        s["r2"], s["h2"], _ = ok(*zk.block_norm(s["r1"], s["d"], norm=zk.ZK_NORM_LAYER, bias=self.gains[0]))
        return s


def test_every_step():
    layer = Layer(1, 96, [1, 5, 17, 40, 3])
    x = torch.randn(5, DIM, generator=layer.gen, device="cuda").to(BF16)
    s = layer.forward(x)
    torch.cuda.synchronize()
    assert layer.fault.item() == 0
    c = {k: v.cpu() for k, v in s.items()}
    gains, gate = [g.cpu() for g in layer.gains], layer.gate.cpu()

    def product(codes, scales, w, dtype):
        return ref.product(codes, w[0].cpu(), scales, w[1].cpu(), dtype)
    codes, scales = ref.codes_of(ref.norm_steps(c["x"], gain=gains[0])[1])
    assert s["r0"] is x
    same(s["h0"], codes)
    same(s["s0"], scales)
    same(s["qkv"], product(c["h0"], c["s0"], layer.qkv, BF16))
    front = layer.prefix.tolist()
    table = [front + row[len(front):] for row in layer.table.tolist()]
    out, lse = check_attention(layer.cache, s["q"], layer.cu.tolist(), layer.lens.tolist(), table, len(front), HEAD ** -0.5)
    assert torch.equal(out, s["a"]) and torch.equal(lse, s["lse"])
    codes, scales = ref.codes_of(c["a"].reshape(5, -1).float())
    same(s["ca"], codes)
    same(s["sa"], scales)
    same(s["o"], product(c["ca"], c["sa"], layer.out, BF16))
    r, h = ref.norm_steps(c["x"], c["o"], gain=gains[1], post_norm=ref.RMS, post_gain=gains[2], gate=gate)
    codes, scales = ref.codes_of(h)
    same(s["r1"], r)
    same(s["h1"], codes)
    same(s["s1"], scales)
    same(s["u"], product(c["h1"], c["s1"], layer.up, F32))
    codes, scales = ref.codes_of(torch.relu(c["u"]))
    same(s["cu"], codes)
    same(s["su"], scales)
    same(s["d"], product(c["cu"], c["su"], layer.down, BF16))
    r, h = ref.norm_steps(c["r1"], c["d"], norm=ref.LAYER, bias=gains[0])
    same(s["r2"], r)
    same(s["h2"], h.to(BF16))


def test_in_a_graph():
    """Captured once; replayed for other inputs, with the program's own work between, it gives what the calls give."""
    layer = Layer(2, 112, [2, 30, 9])
    x = torch.randn(3, DIM, generator=layer.gen, device="cuda").to(BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.forward(x)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = layer.forward(x)
    held = [t.clone() for t in (layer.cache.k, layer.cache.v, layer.cache.k_exp, layer.cache.v_exp)]
    for _ in range(4):
        x.copy_(torch.randn(3, DIM, generator=layer.gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in s.items()}
        for t, w in zip((layer.cache.k, layer.cache.v, layer.cache.k_exp, layer.cache.v_exp), held):
            t.copy_(w)
        want = layer.forward(x)
        for k in got:
            assert torch.equal(got[k], want[k]), k
        for t, w in zip((layer.cache.k, layer.cache.v, layer.cache.k_exp, layer.cache.v_exp), held):
            t.copy_(w)
    assert layer.fault.item() == 0


def test_product_is_proved():
    """The sums that a product gives are the Y of a matmul proof for the same codes, and one that is off by one is not."""
    layer = Layer(3, 64, [1, 2])
    x = torch.randn(20, DIM, generator=layer.gen, device="cuda").to(BF16)
    _, _, codes, _ = zk.block_norm(x, gain=layer.gains[0], quantise=True)
    w = layer.up[0]
    rc, Y = zk.i8_matmul(codes, w, dtype=torch.int32)
    assert rc == zk.ZK_OK
    X, W = codes.to(torch.int16), w.t().contiguous().to(torch.int16)
    seed = b"sums of products of 8-bit codes."
    rc, proof = zk.matmul_sumcheck_prove_i16(seed, X, W)
    assert rc == zk.ZK_OK

    def field(t):
        v = zk.Vec(t.numel())
        assert zk.fr_from_i32(v, t.reshape(-1).to(torch.int32).contiguous()) == zk.ZK_OK
        return v
    assert zk.matmul_sumcheck_verify(seed, proof, 20, DIM, INNER, Y=field(Y), X=field(X), W=field(W)) == zk.ZK_OK
    Y[3, 7] += 1
    assert zk.matmul_sumcheck_verify(seed, proof, 20, DIM, INNER, Y=field(Y), X=field(X), W=field(W)) == zk.ZK_E_REJECT
