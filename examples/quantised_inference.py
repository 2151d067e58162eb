#!/usr/bin/env python3
"""A small quantised decoder that answers, and proofs of the integers it answered with.

Prompts of different lengths go through two layers (4-bit weights, an 8-bit cache of keys and values in pages), then a few
tokens are generated one at a time, each reported with its log probability and alternatives.  Afterwards the cache's codes
are proved to be 8-bit integers (a lookup), and one layer's product with 16-bit activations is proved to be what it is (a
sumcheck), both verified against the tensors.  Weights are random, so are the answers.

    python examples/quantised_inference.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2404_16109_amd as zk  # noqa: E402

VOCAB, DIM, HEADS, KV_HEADS, HEAD_DIM, FFN, LAYERS, GROUP, PAGE, PAGES = 1003, 256, 4, 2, 64, 512, 2, 64, 16, 64


def ok(rc):
    assert rc == zk.ZK_OK, rc


class Linear:
    """outputs x inputs in 4 bits: weights are unit * c * scale, scales 16-bit integers, one to a group of inputs."""

    def __init__(self, gen, outputs, inputs):
        w = torch.randn(outputs, inputs, generator=gen, device="cuda") / inputs ** 0.5
        groups = w.view(outputs, -1, GROUP)
        step = groups.abs().amax(2, keepdim=True) / 7.0
        self.unit = float(step.max()) / 4095.0
        scale = (step / self.unit).round().clamp(1, 4095)
        codes = (groups / (scale * self.unit)).round().clamp(-8, 7).view(outputs, inputs).to(torch.int64) + 8
        self.codes = (codes[:, 0::2] | (codes[:, 1::2] << 4)).to(torch.uint8).contiguous()
        self.scales = scale.view(outputs, -1).to(torch.int16).contiguous()

    def __call__(self, x):
        rc, y = zk.w4_matvec(x.contiguous(), self.codes, self.scales, GROUP, self.unit)
        ok(rc)
        return y


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    def __init__(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.embed = torch.randn(VOCAB, DIM, generator=gen, device="cuda").to(torch.bfloat16)
        self.layers = []
        for _ in range(LAYERS):
            layer = {"qkv": Linear(gen, (HEADS + 2 * KV_HEADS) * HEAD_DIM, DIM), "out": Linear(gen, DIM, HEADS * HEAD_DIM),
                     "up": Linear(gen, FFN, DIM), "down": Linear(gen, DIM, FFN), "cache": zk.KvCache.empty(PAGES, KV_HEADS, PAGE, HEAD_DIM)}
            self.layers.append(layer)
        self.head = Linear(gen, VOCAB, DIM)
        self.fault = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forward(self, tokens, new, lens, table):
        """tokens: the new ones of all sequences, one after the other; new: how many of each; lens: lengths with them.  Returns
        the logits of each sequence's last token."""
        cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
        where = torch.tensor(lens, dtype=torch.int32, device="cuda")
        x = self.embed[tokens]
        for layer in self.layers:
            qkv = layer["qkv"](norm(x)).view(-1, HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
            ok(zk.kvcache_append(layer["cache"], k, v, cu, where, table, max(new), fault=self.fault))
            rc, a, _ = zk.kvcache_attention(layer["cache"], q, cu, where, table, max(new), max(lens), HEAD_DIM ** -0.5, fault=self.fault)
            ok(rc)
            x = x + layer["out"](a.reshape(-1, HEADS * HEAD_DIM))
            x = x + layer["down"](torch.relu(layer["up"](norm(x))))
        last = cu[1:].long() - 1
        return self.head(norm(x[last]))


def generate(model, prompts, steps):
    """Tokens of each sequence after the prompt, and what is reported with each step."""
    lens = [len(p) for p in prompts]
    most = -(-(max(lens) + steps) // PAGE)
    table = torch.arange(len(prompts) * most, dtype=torch.int32, device="cuda").view(len(prompts), most)
    tokens = torch.tensor([t for p in prompts for t in p], device="cuda")
    new, answers, reports = list(lens), [], []
    for _ in range(steps):
        logits = model.forward(tokens, new, lens, table)
        rc, r = zk.logprobs(logits, top=1)
        ok(rc)
        tokens = r["top_ids"][:, 0].long()
        rc, r = zk.logprobs(logits, tokens.to(torch.int32), top=5)
        ok(rc)
        answers.append(tokens)
        reports.append(r)
        new = [1] * len(prompts)
        lens = [n + 1 for n in lens]
    assert model.fault.item() == 0
    return torch.stack(answers, 1), reports, table, [n - 1 for n in lens]


def prove_cache(model, table, length):
    """The keys of a sequence's first tokens, as many as a power of two holds, are integers of 8 bits."""
    rc, k_codes, _ = zk.kvcache_read(model.layers[0]["cache"], table, length, fault=model.fault)
    ok(rc)
    codes = k_codes.reshape(-1)
    X = codes[:1 << (codes.numel().bit_length() - 1)].contiguous()
    T, S = zk.Vec(256), zk.Vec(X.numel())
    ok(zk.fr_from_i32(T, torch.arange(-128, 128, dtype=torch.int32, device="cuda")))
    ok(zk.fr_from_i32(S, X))
    rc, proof, _ = zk.tlookup_prove_small(b"cache codes are 8-bit integers..", X, None, None, X + 128, T)
    ok(rc)
    ok(zk.tlookup_verify(b"cache codes are 8-bit integers..", proof, T, X.numel(), S=S)[0])
    return len(proof)


def prove_product(layer, x):
    """Y = X W for 16-bit activations and the layer's weights as 16-bit integers, Y as the layer computes it."""
    X = (x.float() * 256).round().clamp(-32768, 32767).to(torch.int16)
    rc, Y = zk.w4_matvec(X, layer.codes, layer.scales, GROUP)
    ok(rc)
    rc, W = zk.w4_expand_i16(layer.codes, layer.scales, GROUP)
    ok(rc)
    seed = b"the product is what it should be"
    rc, proof = zk.matmul_sumcheck_prove_i16(seed, X, W)
    ok(rc)

    def field(t):
        """Integers of more than 32 bits in two parts."""
        hi, lo, v = zk.Vec(t.numel()), zk.Vec(t.numel()), zk.Vec(t.numel())
        flat = t.reshape(-1).long()
        ok(zk.fr_from_i32(hi, (flat >> 16).to(torch.int32)))
        ok(zk.fr_from_i32(lo, (flat & 0xffff).to(torch.int32)))
        ok(zk.fr_axpy(v, lo, 1 << 16, hi))
        return v
    ok(zk.matmul_sumcheck_verify(seed, proof, X.shape[0], X.shape[1], W.shape[1], Y=field(Y), X=field(X), W=field(W)))
    return len(proof)


def main():
    model = Decoder(1)
    gen = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, VOCAB, (n,), generator=gen).tolist() for n in (37, 5, 130)]
    answers, reports, table, lens = generate(model, prompts, 6)
    for b, p in enumerate(prompts):
        print("prompt of %d tokens:" % len(p), " ".join("%d (log p %.2f, entropy %.2f)" % (t, reports[i]["target"][b], reports[i]["entropy"][b])
                                                        for i, t in enumerate(answers[b].tolist())))
    print("codes of the cache: a proof of %d bytes" % prove_cache(model, table[2], lens[2]))
    x = norm(model.embed[torch.tensor(prompts[0], device="cuda")])
    print("a product with 4-bit weights: a proof of %d bytes" % prove_product(model.layers[0]["qkv"], x))
    return answers, reports


if __name__ == "__main__":
    main()
