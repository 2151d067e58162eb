"""What the speed of the quantised inference operators is measured on: the cache of 8-bit keys and values with the attention
that reads it, products with 4-bit weights, and the log probabilities an answer is reported with.

A case is one call of a public entry point on device-resident inputs.  The codes in the cache are integers that a lookup
proof is made of, and the product of 16-bit integers is the Y of a matmul proof: those outputs are whole numbers and are
returned as such.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
POISON = -128   # the exponent of a page whose scale is not a number
EXP_MIN, EXP_MAX = -40, 40


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # One new token of each of 32 sequences enters the cache: a step of a served batch, bound by latency.
        {"name": "append_step", "kind": "append", "seqs": 32, "new": 1, "ragged": False, "len": 2048, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16"},
        # Prompts of up to 2048 tokens enter it behind what it holds of a shared beginning, 40 heads of their own keys.
        {"name": "append_prompts", "kind": "append", "seqs": 7, "new": 2048, "ragged": True, "len": 2600, "kv_heads": 40,
         "dim": 128, "page": 64, "dtype": "f16"},
        # The smallest call of a server: one sequence, one token, a few hundred tokens of context, small pages.
        {"name": "attend_one", "kind": "attend", "seqs": 1, "new": 1, "ragged": False, "len": 777, "heads": 40,
         "kv_heads": 8, "dim": 128, "page": 16, "window": 0, "dtype": "bf16"},
        # A step of a served batch: 32 sequences of up to 4096 tokens, five query heads to each head of the cache.
        {"name": "attend_batch", "kind": "attend", "seqs": 32, "new": 1, "ragged": True, "len": 4096, "heads": 40,
         "kv_heads": 8, "dim": 128, "page": 64, "window": 0, "dtype": "bf16"},
        # One long document: the work of a single row has to be spread over the card.
        {"name": "attend_long", "kind": "attend", "seqs": 1, "new": 1, "ragged": False, "len": 131071, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 128, "window": 0, "dtype": "f16"},
        # Four drafted tokens of each of 24 sequences are checked at once, in a model whose heads see the last 1000 tokens.
        {"name": "attend_draft_window", "kind": "attend", "seqs": 24, "new": 4, "ragged": True, "len": 3001, "heads": 16,
         "kv_heads": 4, "dim": 80, "page": 32, "window": 1000, "dtype": "bf16"},
        # A prompt of 2048 tokens through 40 heads: bound by the matrix products.
        {"name": "attend_prompt", "kind": "attend", "seqs": 1, "new": 2048, "ragged": False, "len": 2048, "heads": 40,
         "kv_heads": 40, "dim": 128, "page": 64, "window": 0, "dtype": "bf16"},
        # A projection of a 13B layer (5120 x 5120) for one token.
        {"name": "product_one", "kind": "product", "rows": 1, "n": 5120, "k": 5120, "group": 128, "dtype": "bf16"},
        # The exact integers of a 7B layer's down projection for eight tokens: what a matmul proof is made of.
        {"name": "product_ints", "kind": "product", "rows": 8, "n": 4096, "k": 11008, "group": 32, "dtype": "i16"},
        # The output head of a 32001-token vocabulary for 32 tokens, in 32 bits.
        {"name": "product_head", "kind": "product", "rows": 32, "n": 32001, "k": 5120, "group": 64, "dtype": "f32"},
        # What is reported with one answered token of each of 8 sequences.
        {"name": "logprobs_step", "kind": "logprobs", "rows": 8, "vocab": 32001, "top": 5, "masked": False,
         "dtype": "bf16"},
        # The log probabilities of a whole prompt of 2048 tokens, part of the vocabulary forbidden.
        {"name": "logprobs_prompt", "kind": "logprobs", "rows": 2048, "vocab": 50257, "top": 20, "masked": True,
         "dtype": "f32"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(case, name):
    """Whether a case is no more work than the listed one of that name."""
    a, b = work(case), work(next(c for c in listed() if c["name"] == name))
    return a["bytes"] <= b["bytes"] and a["flops"] <= b["flops"]


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "product", "product", "logprobs"])
    while True:
        if kind == "append":
            new = rng.choice([1, 1, _log_uniform(rng, 2, 2000)])
            seqs = _log_uniform(rng, 1, 64 if new == 1 else max(1, min(64, 12000 // new)))
            case = {"kind": kind, "seqs": seqs, "new": new, "ragged": rng.random() < 0.7, "len": new + _log_uniform(rng, 1, 4000) - 1,
                    "kv_heads": rng.choice([1, 2, 4, 8, 40]), "dim": rng.choice([64, 80, 96, 128, 256]),
                    "page": rng.choice([16, 32, 64, 128]), "dtype": rng.choice(["bf16", "f16", "f32"])}
            if _most(case, "append_prompts"):
                return case
        elif kind == "attend":
            kv = rng.choice([1, 2, 4, 8, 40])
            new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_uniform(rng, 9, 2000)])
            length = new + _log_uniform(rng, 1, 60000 if new <= 8 else 4000) - 1
            case = {"kind": kind, "seqs": _log_uniform(rng, 1, 48), "new": new, "ragged": rng.random() < 0.7, "len": length,
                    "heads": kv * (rng.choice([1, 2, 4, 5, 8]) if kv < 40 else 1), "kv_heads": kv,
                    "dim": rng.choice([64, 80, 96, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128]),
                    "window": rng.choice([0, 0, _log_uniform(rng, 16, 4000)]), "dtype": rng.choice(["bf16", "f16"])}
            # the plain form holds all scores and all keys in 32 bits
            small = case["seqs"] * case["heads"] * new * length < 1 << 28 and case["seqs"] * kv * length * case["dim"] < 1 << 28
            if small and (_most(case, "attend_batch") or _most(case, "attend_prompt")):
                return case
        elif kind == "product":
            case = {"kind": kind, "rows": rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 64)]), "n": _log_uniform(rng, 200, 40000),
                    "k": 32 * _log_uniform(rng, 8, 440), "group": rng.choice([32, 64, 128]),
                    "dtype": rng.choice(["bf16", "f16", "f32", "i16"])}
            if _most(case, "product_head"):
                return case
        else:
            case = {"kind": kind, "rows": _log_uniform(rng, 1, 4096), "vocab": _log_uniform(rng, 1000, 160000), "top": rng.randint(1, 20),
                    "masked": rng.random() < 0.5, "dtype": rng.choice(["bf16", "f16", "f32"])}
            if _most(case, "logprobs_prompt"):
                return case


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)


def _normal(gen, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * scale


def _exponent(amax):
    """The smallest e in [EXP_MIN, EXP_MAX] with amax <= 127 * 2^e, elementwise; POISON where amax is not finite."""
    m, x = torch.frexp(amax)
    e = torch.where(m * 128 <= 127, x - 7, x - 6)
    e = torch.where(amax > 0, e, torch.full_like(e, EXP_MIN)).clamp(EXP_MIN, EXP_MAX)
    return torch.where(torch.isfinite(amax), e, torch.full_like(e, POISON)).to(torch.int8)


def _lengths(case):
    """New tokens and total lengths of the sequences, on the host, from the case alone; of ragged ones some have no new token."""
    B, new, length = case["seqs"], case["new"], case["len"]
    if not case["ragged"]:
        return [new] * B, [length] * B
    g = torch.Generator().manual_seed(B * 100003 + new * 1009 + length)
    n = torch.randint(0 if B > 2 and new > 1 else 1, new + 1, (B,), generator=g).tolist()
    n[0] = new
    lens = [x + int(y * (length - new)) for x, y in zip(n, torch.rand(B, generator=g).tolist())]
    lens[0] = length
    return n, lens


def _sequences(case, seed, gen):
    """The descriptors of a ragged batch, and a cache that holds what each sequence has before its new tokens (of an
    attention case: all of its tokens)."""
    H, d, T = case["kv_heads"], case["dim"], case["page"]
    n, lens = _lengths(case)
    used = [-(-x // T) for x in lens]
    order = torch.randperm(sum(used) + 3, generator=torch.Generator().manual_seed(int(seed) + 3), dtype=torch.int64).to(torch.int32)
    table = torch.full((len(n), max(max(used), 1)), -1, dtype=torch.int32)
    held = torch.arange(table.shape[1])[None, :] < torch.tensor(used)[:, None]
    table[held] = order[:sum(used)]
    pages = sum(used) + 3
    # per page and head a size of its own, as keys have outliers in some heads and tokens
    spread = torch.exp2(torch.randint(-2, 3, (pages, H), generator=gen, device="cuda").float())
    s = {"cu": torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(),
         "table": table.cuda(), "total": sum(n), "max_new": max(n), "max_len": max(lens), "case": case}
    for name in ("k", "v"):
        codes = (_normal(gen, pages, H, T, d) * 36.0).round_().clamp_(-127, 127).to(torch.int8)
        s[name + "_codes"] = codes if name == "k" else codes.transpose(2, 3).contiguous()
        s[name + "_exp"] = _exponent(spread * (4.0 if name == "k" else 2.0))
    return s


def prepare(case, seed):
    gen = _generator(seed)
    kind, dt = case["kind"], DTYPES.get(case["dtype"])
    if kind in ("append", "attend"):
        s = _sequences(case, seed, gen)
        d = case["dim"]
        if kind == "append":
            # keys and values of the new tokens as they leave a joint projection: one row holds the heads of both
            kv = _normal(gen, s["total"], 2, case["kv_heads"], d, scale=1.3).to(dt)
            s["k_new"], s["v_new"] = kv[:, 0], kv[:, 1]
        else:
            s["q"] = _normal(gen, s["total"], case["heads"], d).to(dt)
            s["scale"] = d ** -0.5
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["total"], case["heads"], device="cuda")
        return s
    if kind == "product":
        M, N, K, G = case["rows"], case["n"], case["k"], case["group"]
        s = {"case": case, "group": G}
        s["codes"] = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
        s["scales"] = torch.randint(300, 4096, (N, -(-K // G)), generator=gen, device="cuda", dtype=torch.int16)
        s["unit"] = 2.0 ** -18
        x = _normal(gen, M, K)
        s["x"] = (x * 256).round().clamp(-32768, 32767).to(torch.int16) if case["dtype"] == "i16" else x.to(dt)
        s["out"] = torch.empty(M, N, dtype=torch.int64 if case["dtype"] == "i16" else dt, device="cuda")
        return s
    M, V = case["rows"], case["vocab"]
    x = _normal(gen, M, V, scale=2.5)
    x += 4.0 * (x > 7.0)      # a few likely tokens stand out
    if case["masked"]:
        x[:, torch.rand(V, generator=gen, device="cuda") < 0.2] = -math.inf
    x = x.to(dt)
    targets = torch.randint(0, V, (M,), generator=gen, device="cuda", dtype=torch.int32)
    return {"case": case, "logits": x, "targets": targets, "top": case["top"]}


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"append": _append, "attend": _attend, "product": _product, "logprobs": _logprobs}[kind](state)


def _own(kind, s):
    import paper_2404_16109_amd as zk
    # what a serving program makes once and keeps: the cache's descriptor, and a workspace
    if kind in ("append", "attend"):
        if "cache" not in s:
            s["cache"] = zk.KvCache(s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"])
        if kind == "append":
            rc = zk.kvcache_append(s["cache"], s["k_new"], s["v_new"], s["cu"], s["lens"], s["table"], s["max_new"])
            assert rc == zk.ZK_OK, rc
            return [s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"]]
        if "ws" not in s:
            need = zk.kvcache_attention_workspace_bytes(s["lens"].numel(), s["total"], s["max_new"], s["q"].shape[1],
                                                        s["k_exp"].shape[1], s["q"].shape[2], s["max_len"])
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        rc, out, lse = zk.kvcache_attention(s["cache"], s["q"], s["cu"], s["lens"], s["table"], s["max_new"], s["max_len"],
                                            s["scale"], window=s["case"]["window"], out=s["out"], lse=s["lse"], ws=s["ws"])
        assert rc == zk.ZK_OK, rc
        return [out, lse]
    if kind == "product":
        if "ws" not in s:
            need = zk.w4_matvec_workspace_bytes(s["x"].dtype, *s["x"].shape)
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        rc, y = zk.w4_matvec(s["x"], s["codes"], s["scales"], s["group"], s["unit"], out=s["out"], ws=s["ws"])
        assert rc == zk.ZK_OK, rc
        return y
    if "ws" not in s:
        s["ws"] = torch.empty(max(zk.logprobs_workspace_bytes(*s["logits"].shape, s["top"]), 1), dtype=torch.uint8, device="cuda")
    rc, got = zk.logprobs(s["logits"], s["targets"], s["top"], ws=s["ws"])
    assert rc == zk.ZK_OK, rc
    return got


def _scale_of(exp):
    e = exp.float()
    return torch.where(exp == POISON, torch.full_like(e, math.nan), torch.exp2(e))


def _append_to(new, codes, exps, keep, pages, which, slot, fresh):
    """codes: [pages, heads, tokens, dim], exps: [pages, heads]; both are updated in place at the given pages."""
    x = new.float()[keep]
    size = x.abs().amax(-1)
    size = torch.where(torch.isfinite(x).all(-1), size, torch.full_like(size, math.inf))
    amax = torch.zeros(pages.shape[0], exps.shape[1], device="cuda").index_reduce_(0, which, size, "amax")
    need, held = _exponent(amax).int(), exps[pages].int()
    held = torch.where(fresh[:, None], torch.full_like(held, EXP_MIN), held)
    e = torch.where((need == POISON) | (held == POISON), torch.full_like(need, POISON), torch.maximum(need, held))
    shift = torch.where(e != POISON, held - e, torch.zeros_like(e))
    grown = torch.round(codes[pages].float() * torch.exp2(shift.float())[:, :, None, None])
    grown = grown.masked_fill_(fresh[:, None, None, None], 0.0).to(torch.int8)
    fine = (e != POISON)[which][:, :, None]
    step = torch.exp2(-e.float())[which][:, :, None]
    got = torch.where(fine, torch.round(torch.where(fine, x, torch.zeros_like(x)) * step).clamp(-127, 127), torch.zeros_like(x))
    grown[which, :, slot] = got.to(torch.int8)
    codes[pages] = grown
    exps[pages] = e.to(torch.int8)


def _append(s):
    """Every page that new tokens fall into: its exponent is the larger of what its tokens so far and the new ones need,
    the codes it holds are rounded to it, and the new tokens' codes are written.  A page that begins is cleared first."""
    cu, lens, table = s["cu"].long(), s["lens"].long(), s["table"].long()
    T = s["k_codes"].shape[2]
    token = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(cu, token, right=True) - 1
    pos = lens[seq] - (cu[seq + 1] - token)
    keep = pos >= 0
    seq, pos = seq[keep], pos[keep]
    slot = pos % T
    pages, which = torch.unique(table[seq, pos // T], return_inverse=True)
    fresh = torch.zeros(pages.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, which[slot == 0], True)
    where = (keep, pages, which, slot, fresh)
    _append_to(s["k_new"], s["k_codes"], s["k_exp"], *where)
    _append_to(s["v_new"], s["v_codes"].transpose(2, 3), s["v_exp"], *where)
    return [s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"]]


def _attend(s):
    """softmax(scale * q k^T) v over the keys a query sees: those up to its own position, the last `window` of them."""
    cu, lens, table = s["cu"].long(), s["lens"].long(), s["table"].long().clamp(min=0)
    B, q = table.shape[0], s["q"].float()
    Hq, d = q.shape[1:]
    H, T = s["k_codes"].shape[1:3]
    G, n, L = Hq // H, s["max_new"], table.shape[1] * T
    k = (s["k_codes"][table].float() * _scale_of(s["k_exp"])[table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, H, L, d)
    v = (s["v_codes"][table].float() * _scale_of(s["v_exp"])[table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, H, L, d)
    i, j = torch.arange(n, device="cuda"), torch.arange(L, device="cuda")
    new = cu[1:] - cu[:-1]
    rows = (cu[:-1, None] + i).clamp(max=max(s["total"] - 1, 0))
    dense = q[rows].reshape(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, d)
    scores = torch.matmul(dense, k.transpose(2, 3).contiguous()) * s["scale"]
    pos = (lens - new)[:, None] + i
    seen = j <= pos[..., None]
    if s["case"]["window"]:
        seen = seen & (j > pos[..., None] - s["case"]["window"])
    scores = scores.reshape(B, H, G, n, L).masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = torch.where((j < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    out = torch.matmul(p.reshape(B, H, G * n, L), v).reshape(B, H, G, n, d) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + torch.log(total))[..., 0]
    token = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(cu, token, right=True) - 1
    at = token - cu[seq]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, d)[seq, at]
    lse = lse.permute(0, 3, 1, 2).reshape(B, n, Hq)[seq, at]
    return [out.to(s["q"].dtype), lse]


def _weights(s, dtype):
    """c * s as [N, K]: codes lie two to a byte, the lower half first, as c + 8."""
    c = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=-1).reshape(s["codes"].shape[0], -1).to(dtype) - 8
    return c * s["scales"].to(dtype).repeat_interleave(s["group"], dim=1)[:, :c.shape[1]]


def _product(s):
    x = s["x"]
    if x.dtype == torch.int16:
        # whole numbers below 2^53 at every step
        return torch.matmul(x.double(), _weights(s, torch.float64).t()).to(torch.int64)
    return (torch.matmul(x.float(), _weights(s, torch.float32).t()) * s["unit"]).to(x.dtype)


def _logprobs(s):
    x, t = s["logits"].float(), s["targets"].long()[:, None]
    top = x.amax(-1, keepdim=True)
    base = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(x - base)
    total = e.sum(-1, keepdim=True)
    lse = base + torch.log(total)
    entropy = torch.log(total) - torch.where(e > 0, e * (x - base), torch.zeros_like(e)).sum(-1, keepdim=True) / total
    xt = x.gather(1, t)
    index = torch.arange(x.shape[1], device="cuda")
    rank = ((x > xt) | ((x == xt) & (index < t))).sum(-1)
    value, which = torch.sort(x, dim=-1, descending=True, stable=True)
    k = s["top"]
    return {"target": (xt - lse)[:, 0], "rank": rank.to(torch.int32), "lse": lse[:, 0], "entropy": entropy[:, 0],
            "top_ids": which[:, :k].to(torch.int32), "top": value[:, :k] - lse}


# ---- in 64 bits --------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "append":
        return _exact_append(s)
    if kind == "attend":
        return _exact_attend(s)
    if kind == "product":
        return _exact_product(s)
    return _exact_logprobs(s)


def _exact_append(s):
    """Page by page of each sequence, one head at a time taken together."""
    k, v, ke, ve = (s[x].clone() for x in ("k_codes", "v_codes", "k_exp", "v_exp"))
    T = k.shape[2]
    cu, lens, table = s["cu"].tolist(), s["lens"].tolist(), s["table"].tolist()
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        first = lens[b] - n
        for p in range(first // T, -(-lens[b] // T)):
            lo, hi = max(first, p * T), min(lens[b], (p + 1) * T)
            if hi <= lo:
                continue
            page, rows = table[b][p], slice(cu[b] + lo - first, cu[b] + hi - first)
            for new, codes, exps, across in ((s["k_new"], k, ke, False), (s["v_new"], v, ve, True)):
                x = new[rows].double().transpose(0, 1)                                  # heads, tokens, dim
                amax = x.abs().amax((1, 2))
                need = torch.ceil(torch.log2(amax / 127.0).clamp(-60, 60))
                need = need + (amax > 127.0 * torch.exp2(need)).double() - (amax <= 127.0 * torch.exp2(need - 1)).double()
                need = need.clamp(EXP_MIN, EXP_MAX)
                held = exps[page].double() if lo > p * T else torch.full_like(need, EXP_MIN)
                e = torch.maximum(need, held)
                at = codes[page].transpose(1, 2) if across else codes[page]             # heads, tokens, dim
                at.copy_(torch.round(at.double() * torch.exp2(held - e)[:, None, None]) if lo > p * T else torch.zeros_like(at))
                at[:, lo - p * T:hi - p * T] = torch.round(x * torch.exp2(-e)[:, None, None]).clamp(-127, 127).to(torch.int8)
                exps[page] = e.to(torch.int8)
    return [k, v, ke, ve]


def _exact_attend(s):
    """One sequence and one head of the cache after the other, the softmax by its definition."""
    q, T, W = s["q"].double(), s["k_codes"].shape[2], s["case"]["window"]
    Hq, d = q.shape[1:]
    H = s["k_codes"].shape[1]
    G = Hq // H
    out = torch.zeros(q.shape[0], Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((q.shape[0], Hq), -math.inf, dtype=torch.float64, device="cuda")
    cu, lens = s["cu"].tolist(), s["lens"].tolist()
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        if n == 0 or lens[b] == 0:
            continue
        pages = s["table"][b, :-(-lens[b] // T)].long()
        pos = torch.arange(lens[b] - n, lens[b], device="cuda")[:, None]
        j = torch.arange(lens[b], device="cuda")
        hidden = (j > pos) | ((j <= pos - W) if W else (j < 0))
        for h in range(H):
            k = (s["k_codes"][pages, h].double() * torch.exp2(s["k_exp"][pages, h].double())[:, None, None]).reshape(-1, d)[:lens[b]]
            v = s["v_codes"][pages, h].double() * torch.exp2(s["v_exp"][pages, h].double())[:, None, None]
            v = v.transpose(1, 2).reshape(-1, d)[:lens[b]]
            for g in range(G):
                z = (q[cu[b]:cu[b + 1], h * G + g] @ k.t().contiguous()) * s["scale"]
                z = z.masked_fill(hidden, -math.inf)
                some = ~hidden.all(1)
                lse[cu[b]:cu[b + 1], h * G + g] = torch.logsumexp(z, 1)
                w = torch.softmax(z[some], 1)
                at = torch.arange(cu[b], cu[b + 1], device="cuda")[some]
                out[at, h * G + g] = w @ v
    return [out, lse]


def _exact_product(s):
    if s["x"].dtype == torch.int16:
        return None
    x = s["x"].double()
    N, half = s["codes"].shape
    y = torch.zeros(x.shape[0], N, dtype=torch.float64, device="cuda")
    G = s["group"]
    for g in range(s["scales"].shape[1]):
        b = s["codes"][:, g * G // 2:(g + 1) * G // 2]
        xs = x[:, g * G:(g + 1) * G]
        part = xs[:, 0::2] @ ((b & 15).double() - 8).t().contiguous() + xs[:, 1::2] @ ((b >> 4).double() - 8).t().contiguous()
        y += part * s["scales"][:, g].double()
    return y * s["unit"]


def _exact_logprobs(s):
    x = s["logits"]
    M, k = x.shape[0], s["top"]
    got = {"target": [], "rank": None, "lse": [], "entropy": [], "top_ids": None, "top": []}
    for at in range(0, M, 256):
        y = x[at:at + 256].double()
        p = torch.log_softmax(y, 1)
        got["lse"].append(torch.logsumexp(y, 1))
        got["target"].append(p.gather(1, s["targets"][at:at + 256].long()[:, None])[:, 0])
        got["entropy"].append(-(torch.exp(p) * p.nan_to_num(neginf=0.0)).sum(1))
        got["top"].append(torch.topk(p, k, dim=1).values)
    return {name: None if parts is None else torch.cat(parts) for name, parts in got.items()}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f32": 4, "f16": 2, "bf16": 2, "i16": 2}[case["dtype"]]
    if kind == "append":
        # the new tokens read and their codes written
        values = _tokens(case) * case["kv_heads"] * case["dim"] * 2
        return {"bytes": values * (size + 1), "flops": 3 * values}
    if kind == "attend":
        pairs, keys = _pairs(case)
        values = _tokens(case) * case["heads"] * case["dim"]
        return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] + 2 * values * size + _tokens(case) * case["heads"] * 4,
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    if kind == "product":
        M, N, K = case["rows"], case["n"], case["k"]
        out = 8 if case["dtype"] == "i16" else size
        return {"bytes": N * K // 2 + 2 * N * -(-K // case["group"]) + M * K * size + M * N * out, "flops": 2 * M * N * K}
    M, V = case["rows"], case["vocab"]
    return {"bytes": M * V * size + M * (20 + 8 * case["top"]), "flops": 5 * M * V}


def _tokens(case):
    return sum(_lengths(case)[0])


def _pairs(case):
    """(pairs of a query and a key it sees, keys that are seen)."""
    n, lens = (torch.tensor(x, dtype=torch.float64) for x in _lengths(case))
    if not case["window"]:
        return float((n * (lens - (n - 1) / 2)).sum()), float(lens[n > 0].sum())
    W, i = case["window"], torch.arange(case["new"])
    pos = (lens - n)[:, None] + i                     # a query sees min(W, pos + 1) keys
    pairs = torch.where(i < n[:, None], (pos + 1).clamp(max=W), torch.zeros_like(pos)).sum()
    return float(pairs), float(torch.minimum(lens, n + W - 1)[n > 0].sum())
