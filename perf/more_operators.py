"""What the speed of a decoder layer in 8 bits is measured on: what stands between two blocks (residual, norms, gate, codes),
activations as codes, products of 8-bit integers, and attention for a batch behind a prompt that all of it shares.

A case is one call of a public entry point on device-resident inputs.  The codes of activations and the sums of their products
are integers that proofs are made of, and are defined bit for bit: those outputs are whole numbers and are returned as such.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i32": torch.int32}


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # Between two blocks of a 13B layer, one token of one sequence: bound by latency.
        {"name": "norm_step", "kind": "norm", "rows": 1, "dim": 5120, "norm": "rms", "post": "none", "block": True,
         "gate": "none", "alpha": 1.0, "codes": True, "dtype": "bf16"},
        # Layer norms in 32 bits of a ragged batch of an odd width, residual scaled, a gate for each channel.
        {"name": "norm_odd", "kind": "norm", "rows": 777, "dim": 4097, "norm": "layer", "post": "none", "block": True,
         "gate": "channel", "alpha": 0.7, "codes": False, "dtype": "f32"},
        # A prompt of 8192 tokens: norms on both sides of the residual, a gate for each token and channel, codes for the next product.
        {"name": "norm_prompt", "kind": "norm", "rows": 8192, "dim": 5120, "norm": "rms", "post": "rms", "block": True,
         "gate": "token", "alpha": 1.0, "codes": True, "dtype": "bf16"},
        # The inner activations of a 13B layer for a step of a served batch.
        {"name": "quantise_step", "kind": "quantise", "rows": 32, "dim": 13824, "dtype": "bf16"},
        # The same for a prompt of 8192 tokens.
        {"name": "quantise_prompt", "kind": "quantise", "rows": 8192, "dim": 13824, "dtype": "f16"},
        # A projection of a 13B layer for one token.
        {"name": "matmul_one", "kind": "matmul", "rows": 1, "n": 5120, "k": 5120, "dtype": "bf16"},
        # Its up projection for a step of a served batch.
        {"name": "matmul_batch", "kind": "matmul", "rows": 32, "n": 13824, "k": 5120, "dtype": "f16"},
        # The exact integers of its down projection for some hundred tokens: what a matmul proof is made of.
        {"name": "matmul_ints", "kind": "matmul", "rows": 333, "n": 5120, "k": 13824, "dtype": "i32"},
        # Its up projection for a prompt of 8192 tokens: bound by the matrix cores.
        {"name": "matmul_prompt", "kind": "matmul", "rows": 8192, "n": 13824, "k": 5120, "dtype": "bf16"},
        # Four short answers behind one instruction of 2032 tokens, small pages, heads of 80.
        {"name": "prefix_few", "kind": "prefix", "seqs": 4, "new": 1, "ragged": True, "prefix": 2032, "own": 100, "heads": 16,
         "kv_heads": 4, "dim": 80, "page": 16, "dtype": "f16"},
        # A step of 64 sequences behind one document of 8192 tokens.
        {"name": "prefix_step", "kind": "prefix", "seqs": 64, "new": 1, "ragged": True, "prefix": 8192, "own": 512, "heads": 40,
         "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # Questions of up to 64 tokens, 16 at once, about a document of 32768 tokens.
        {"name": "prefix_questions", "kind": "prefix", "seqs": 16, "new": 64, "ragged": True, "prefix": 32768, "own": 300,
         "heads": 40, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _most(case, name):
    """Whether a case is no more work than the listed one of that name."""
    a, b = work(case), work(next(c for c in listed() if c["name"] == name))
    return a["bytes"] <= b["bytes"] and a["flops"] <= b["flops"]


def draw(rng):
    kind = rng.choice(["norm", "norm", "quantise", "matmul", "matmul", "matmul", "prefix", "prefix"])
    while True:
        if kind == "norm":
            block = rng.random() < 0.8
            case = {"kind": kind, "rows": _log_uniform(rng, 1, 16384), "dim": _log_uniform(rng, 64, 16384), "norm": rng.choice(["rms", "layer"]),
                    "post": rng.choice(["none", "rms", "layer"]) if block else "none", "block": block,
                    "gate": rng.choice(["none", "channel", "token"]) if block else "none", "alpha": rng.choice([1.0, 0.5, 1.7]),
                    "codes": rng.random() < 0.6, "dtype": rng.choice(["bf16", "f16", "f32"])}
            if rng.random() < 0.5:
                case["dim"] = -(-case["dim"] // 64) * 64
            if _most(case, "norm_prompt"):
                return case
        elif kind == "quantise":
            case = {"kind": kind, "rows": _log_uniform(rng, 1, 16384), "dim": _log_uniform(rng, 64, 30000), "dtype": rng.choice(["bf16", "f16", "f32"])}
            if rng.random() < 0.6:
                case["dim"] = -(-case["dim"] // 64) * 64
            if _most(case, "quantise_prompt"):
                return case
        elif kind == "matmul":
            case = {"kind": kind, "rows": rng.choice([1, rng.randint(2, 32), _log_uniform(rng, 33, 600), _log_uniform(rng, 600, 8192)]),
                    "n": _log_uniform(rng, 200, 40000), "k": 16 * _log_uniform(rng, 16, 1700), "dtype": rng.choice(["bf16", "f16", "f32", "i32"])}
            if _most(case, "matmul_prompt"):
                return case
        else:
            kv, page = rng.choice([1, 2, 4, 8, 40]), rng.choice([16, 32, 64, 128])
            new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_uniform(rng, 9, 200)])
            case = {"kind": kind, "seqs": _log_uniform(rng, 2, 128 if new <= 8 else 16), "new": new, "ragged": rng.random() < 0.7,
                    "prefix": page * max(1, _log_uniform(rng, 128, 60000) // page), "own": new + _log_uniform(rng, 1, 2000) - 1,
                    "heads": kv * (rng.choice([1, 2, 4, 5, 8]) if kv < 40 else 1), "kv_heads": kv,
                    "dim": rng.choice([64, 80, 96, 128, 128, 256]), "page": page, "dtype": rng.choice(["bf16", "f16"])}
            # the plain form holds all scores and all keys in 32 bits
            small = (case["seqs"] * case["heads"] * new * (case["prefix"] + case["own"]) < 1 << 30
                     and kv * (case["prefix"] + case["seqs"] * case["own"]) * case["dim"] < 1 << 28)
            if small and _most(case, "prefix_questions"):
                return case


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)


def _normal(gen, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * scale


def _activations(gen, rows, dim, dtype, scale=1.0):
    """As they are in a trained model: a few channels many times larger than the others, tokens of unlike size."""
    x = _normal(gen, rows, dim, scale=scale)
    x *= 1.0 + 20.0 * (torch.rand(dim, generator=gen, device="cuda") < 0.002)
    x *= 0.5 + torch.rand(rows, 1, generator=gen, device="cuda")
    return x.to(dtype)


def _codes(gen, rows, dim):
    return _normal(gen, rows, dim, scale=36.0).round_().clamp_(-127, 127).to(torch.int8)


def _lengths(case):
    """New tokens of the sequences, and their total lengths with the prefix, on the host, from the case alone."""
    B, new, P, length = case["seqs"], case["new"], case["prefix"], case["own"]
    if not case["ragged"]:
        return [new] * B, [P + length] * B
    g = torch.Generator().manual_seed(B * 100003 + new * 1009 + length)
    n = torch.randint(0 if B > 2 and new > 1 else 1, new + 1, (B,), generator=g).tolist()
    n[0] = new
    lens = [P + x + int(y * (length - new)) for x, y in zip(n, torch.rand(B, generator=g).tolist())]
    lens[0] = P + length
    return n, lens


def _sequences(case, seed, gen):
    """A ragged batch, the pages of the prefix that it shares, and a cache that holds all tokens."""
    H, d, T, P = case["kv_heads"], case["dim"], case["page"], case["prefix"]
    n, lens = _lengths(case)
    shared = P // T
    used = [-(-x // T) - shared for x in lens]
    pages = shared + sum(used) + 3
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed) + 3), dtype=torch.int64).to(torch.int32)
    table = torch.full((len(n), shared + max(max(used), 1)), -1, dtype=torch.int32)
    at = torch.arange(table.shape[1])[None, :] - shared
    table[(at >= 0) & (at < torch.tensor(used)[:, None])] = order[shared:shared + sum(used)]
    # per page and head a size of its own, as keys have outliers in some heads and tokens
    spread = torch.randint(-6, -2, (pages, H), generator=gen, device="cuda", dtype=torch.int8)
    s = {"case": case, "cu": torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(),
         "table": table.cuda(), "shared": order[:shared].cuda(), "total": sum(n), "max_new": max(n), "max_len": max(lens),
         "k_exp": spread, "v_exp": spread - 1}
    s["k_codes"] = _codes(gen, pages * H * T, d).reshape(pages, H, T, d)
    s["v_codes"] = _codes(gen, pages * H * d, T).reshape(pages, H, d, T)
    return s


def prepare(case, seed):
    gen = _generator(seed)
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "prefix":
        s = _sequences(case, seed, gen)
        s["q"] = _normal(gen, s["total"], case["heads"], case["dim"]).to(dt)
        s["scale"] = case["dim"] ** -0.5
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["total"], case["heads"], device="cuda")
        return s
    if kind == "matmul":
        M, N, K = case["rows"], case["n"], case["k"]
        return {"case": case, "x": _codes(gen, M, K), "w": _codes(gen, N, K),
                "x_scales": 0.01 + 0.03 * torch.rand(M, generator=gen, device="cuda"),
                "w_scales": 0.0002 + 0.0006 * torch.rand(N, generator=gen, device="cuda"),
                "out": torch.empty(M, N, dtype=dt, device="cuda")}
    M, D = case["rows"], case["dim"]
    s = {"case": case, "x": _activations(gen, M, D, dt)}
    if kind == "quantise" or case["codes"]:
        s["h"], s["scales"] = torch.empty(M, D, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    if kind == "quantise":
        return s
    s["eps"] = 1e-5
    s["gain"] = (1.0 + 0.2 * _normal(gen, D)).to(dt)
    s["bias"] = _normal(gen, D, scale=0.1).to(dt) if case["norm"] == "layer" else None
    s["z"] = _activations(gen, M, D, dt, scale=0.6) if case["block"] else None
    s["post_gain"] = (0.5 + 0.1 * _normal(gen, D)).to(dt) if case["post"] != "none" else None
    s["gate"] = {"none": lambda: None, "channel": lambda: _normal(gen, D, scale=0.5).to(dt),
                 "token": lambda: _normal(gen, M, D, scale=0.5).to(dt)}[case["gate"]]()
    s["r"] = torch.empty_like(s["x"])
    if not case["codes"]:
        s["h"], s["scales"] = torch.empty_like(s["x"]), None
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"norm": _norm, "quantise": _quantise, "matmul": _matmul, "prefix": _prefix}[kind](state)


def _own(kind, s):
    import paper_2404_16109_amd as zk
    # what a serving program makes once and keeps: the cache's descriptor, and a workspace
    if kind == "norm":
        norms = {"none": zk.ZK_NORM_NONE, "rms": zk.ZK_NORM_RMS, "layer": zk.ZK_NORM_LAYER}
        c = s["case"]
        rc, r, h, scales = zk.block_norm(s["x"], s["z"], norm=norms[c["norm"]], gain=s["gain"], bias=s["bias"], eps=s["eps"],
                                         post_norm=norms[c["post"]], post_gain=s["post_gain"], gate=s["gate"], alpha=c["alpha"],
                                         r=s["r"], h=s["h"], scales=s["scales"])
        assert rc == zk.ZK_OK, rc
        return {"r": r, "h": h, "scales": scales} if c["codes"] else {"r": r, "h": h}
    if kind == "quantise":
        rc, codes, scales = zk.i8_quantise(s["x"], codes=s["h"], scales=s["scales"])
        assert rc == zk.ZK_OK, rc
        return {"codes": codes, "scales": scales}
    if kind == "matmul":
        if "ws" not in s:
            need = zk.i8_matmul_workspace_bytes(s["x"].shape[0], *s["w"].shape)
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        rc, y = zk.i8_matmul(s["x"], s["w"], s["x_scales"], s["w_scales"], out=s["out"], ws=s["ws"])
        assert rc == zk.ZK_OK, rc
        return y
    if "cache" not in s:
        s["cache"] = zk.KvCache(s["k_codes"], s["v_codes"], s["k_exp"], s["v_exp"])
        need = zk.kvcache_attention_prefix_workspace_bytes(s["lens"].numel(), s["total"], s["max_new"], s["q"].shape[1], s["k_exp"].shape[1],
                                                           s["q"].shape[2], s["case"]["prefix"], s["max_len"])
        s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    rc, out, lse = zk.kvcache_attention_prefix(s["cache"], s["q"], s["cu"], s["lens"], s["table"], s["shared"], s["max_new"], s["max_len"],
                                               s["scale"], out=s["out"], lse=s["lse"], ws=s["ws"])
    assert rc == zk.ZK_OK, rc
    return [out, lse]


def _normed(x, norm, gain, bias, eps):
    """Statistics in 64 bits, rounded to 32; then one rounding to 32 bits a step."""
    if norm != "none":
        wide = x.double()
        if norm == "layer":
            wide = wide - wide.mean(-1, keepdim=True)
            x = x - x.double().mean(-1, keepdim=True).float()
        x = x * (1.0 / torch.sqrt((wide * wide).mean(-1, keepdim=True) + eps)).float()
    if gain is not None:
        x = x * gain.float()
    return x if bias is None else x + bias.float()


def _coded(h):
    """scale = amax / 127 and codes rint(h * (127 / amax)), the quotients taken in 64 bits and rounded to 32; a row of next to
    nothing is zeros, one that is not finite has no scale."""
    amax = h.abs().amax(-1, keepdim=True)
    some = (amax >= 2.0 ** -100) & torch.isfinite(amax)
    wide = torch.where(some, amax, torch.ones_like(amax)).double()
    codes = torch.where(some, torch.round(h * (127.0 / wide).float()), torch.zeros_like(h)).to(torch.int8)
    scales = torch.where(some, (wide / 127.0).float(), torch.where(amax < 1.0, 0.0, math.nan))
    return codes, scales[:, 0]


def _norm(s):
    c, dt = s["case"], s["x"].dtype
    r = s["x"].float() * c["alpha"]
    if s["z"] is not None:
        t = _normed(s["z"].float(), c["post"], s["post_gain"], None, s["eps"])
        r = r + (t if s["gate"] is None else s["gate"].float() * t)
    r = r.to(dt)
    h = _normed(r.float(), c["norm"], s["gain"], s["bias"], s["eps"])
    if not c["codes"]:
        return {"r": r, "h": h.to(dt)}
    codes, scales = _coded(h)
    return {"r": r, "h": codes, "scales": scales}


def _quantise(s):
    codes, scales = _coded(s["x"].float())
    return {"codes": codes, "scales": scales}


def _matmul(s):
    x, w, out = s["x"], s["w"], s["out"]
    if out.dtype == torch.int32:
        # whole numbers below 2^53 at every step
        return torch.matmul(x.double(), w.double().t()).to(torch.int32)
    return (torch.matmul(x.float(), w.float().t()) * s["x_scales"][:, None] * s["w_scales"]).to(out.dtype)


def _prefix(s):
    """softmax(scale * q k^T) v over the keys up to a query's own position: those of the prefix, computed once for all rows,
    and its sequence's own."""
    c, cu, lens, total = s["case"], s["cu"].long(), s["lens"].long(), s["total"]
    q, P, T = s["q"].float(), c["prefix"], c["page"]
    Hq, d = q.shape[1:]
    H, B, n = c["kv_heads"], lens.shape[0], s["max_new"]
    G = Hq // H
    own_pages = s["table"][:, P // T:].long().clamp(min=0)
    L = own_pages.shape[1] * T
    token = torch.arange(total, device="cuda")
    seq = torch.searchsorted(cu, token, right=True) - 1
    at = token - cu[seq]
    pos = lens[seq] - (cu[seq + 1] - token)
    kx, vx = torch.exp2(s["k_exp"].float())[..., None, None], torch.exp2(s["v_exp"].float())[..., None, None]

    def keys(pages):
        k, v = s["k_codes"][pages].float() * kx[pages], s["v_codes"][pages].float() * vx[pages]
        return k.transpose(-4, -3).flatten(-3, -2), v.transpose(-4, -3).transpose(-2, -1).flatten(-3, -2)

    k, v = keys(s["shared"].long())                                     # heads, prefix, dim
    rows = q.reshape(total, H, G, d).transpose(0, 1).reshape(H, total * G, d)
    shared = (torch.matmul(rows, k.transpose(1, 2).contiguous()) * s["scale"]).reshape(H, total, G, P)
    shared = shared.masked_fill_((torch.arange(P, device="cuda") > pos[:, None])[None, :, None], -math.inf)
    ko, vo = keys(own_pages)                                            # sequences, heads, own, dim
    dense = torch.zeros(B, n, H, G, d, device="cuda")
    dense[seq, at] = q.reshape(total, H, G, d)
    dense = dense.permute(0, 2, 1, 3, 4).reshape(B, H, n * G, d)
    mine = (torch.matmul(dense, ko.transpose(2, 3).contiguous()) * s["scale"]).reshape(B, H, n, G, L)
    first = (lens - (cu[1:] - cu[:-1]))[:, None] + torch.arange(n, device="cuda")
    hidden = P + torch.arange(L, device="cuda") > first[..., None]
    mine = mine.masked_fill_(hidden[:, None, :, None], -math.inf)
    mine_top = mine.amax(-1, keepdim=True).transpose(1, 2)[seq, at].transpose(0, 1)      # heads, rows, group, 1
    top = torch.maximum(shared.amax(-1, keepdim=True), mine_top)
    shared = torch.exp(shared - top)
    there = torch.zeros(B, n, H, G, 1, device="cuda")
    there[seq, at] = top.transpose(0, 1)
    mine = torch.exp(mine - there.transpose(1, 2).reshape(B, n, H, G, 1).reshape(B, H, n, G, 1))
    vo = torch.where((P + torch.arange(L, device="cuda") < lens[:, None])[:, None, :, None], vo, torch.zeros_like(vo))
    o = torch.matmul(mine.reshape(B, H, n * G, L), vo).reshape(B, H, n, G, d).transpose(1, 2)[seq, at].transpose(0, 1)
    o = o + torch.matmul(shared.reshape(H, total * G, P), v).reshape(H, total, G, d)
    weight = shared.sum(-1, keepdim=True) + mine.sum(-1, keepdim=True).transpose(1, 2)[seq, at].transpose(0, 1)
    out = (o / weight).transpose(0, 1).reshape(total, Hq, d)
    lse = (top + torch.log(weight))[..., 0].transpose(0, 1).reshape(total, Hq)
    return [out.to(s["q"].dtype), lse]


# ---- in 64 bits --------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "quantise":
        return {"codes": None, "scales": torch.linalg.vector_norm(s["x"].double(), ord=math.inf, dim=1) / 127}
    if kind == "matmul":
        return _exact_matmul(s)
    return _exact_prefix(s)


def _exact_norm(s):
    c = s["case"]

    def norm(x, how, gain, bias):
        if how == "rms":
            x = x * torch.rsqrt(x.square().mean(1) + s["eps"])[:, None]
        elif how == "layer":
            var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
            x = (x - mean) * torch.rsqrt(var + s["eps"])
        if gain is not None:
            x = x * gain.double()
        return x + bias.double() if bias is not None else x

    alpha = float(torch.tensor(c["alpha"], dtype=torch.float32))   # the call takes it in 32 bits
    r = alpha * s["x"].double()
    if s["z"] is not None:
        t = norm(s["z"].double(), c["post"], s["post_gain"], None)
        r = r + (1.0 if s["gate"] is None else s["gate"].double()) * t
    # the next block sees the residual stream as it is stored
    h = norm(r.to(s["x"].dtype).double(), c["norm"], s["gain"], s["bias"])
    if c["codes"]:
        return {"r": r, "h": None, "scales": h.abs().max(1).values / 127}
    return {"r": r, "h": h}


def _exact_matmul(s):
    """Sums of whole numbers, exact in 64 bits, some outputs at a time."""
    if s["out"].dtype == torch.int32:
        return None
    x = s["x"].double() * s["x_scales"].double()[:, None]
    y = torch.empty(x.shape[0], s["w"].shape[0], dtype=torch.float64, device="cuda")
    for i in range(0, s["w"].shape[0], 2048):
        w = s["w"][i:i + 2048].double().t().contiguous()
        y[:, i:i + 2048] = (x @ w) * s["w_scales"][i:i + 2048].double()
    return y


def _exact_prefix(s):
    """One sequence and one head of the cache after the other, the softmax by its definition."""
    c, q, T = s["case"], s["q"].double(), s["case"]["page"]
    Hq, d = q.shape[1:]
    H, shared = c["kv_heads"], s["shared"].numel()
    G = Hq // H
    out = torch.zeros(q.shape[0], Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((q.shape[0], Hq), -math.inf, dtype=torch.float64, device="cuda")
    cu, lens = s["cu"].tolist(), s["lens"].tolist()

    def numbers(pages, h):
        k = s["k_codes"][pages, h].double() * torch.exp2(s["k_exp"][pages, h].double())[:, None, None]
        v = s["v_codes"][pages, h].double() * torch.exp2(s["v_exp"][pages, h].double())[:, None, None]
        return k.reshape(-1, d), v.transpose(1, 2).reshape(-1, d)

    for h in range(H):
        front = numbers(s["shared"].long(), h)
        for b in range(len(lens)):
            n = cu[b + 1] - cu[b]
            if n == 0:
                continue
            behind = numbers(s["table"][b, shared:-(-lens[b] // T)].long(), h)
            k, v = (torch.cat(x)[:lens[b]] for x in zip(front, behind))
            hidden = torch.arange(lens[b], device="cuda") > torch.arange(lens[b] - n, lens[b], device="cuda")[:, None]
            for g in range(h * G, h * G + G):
                z = ((q[cu[b]:cu[b + 1], g] @ k.t().contiguous()) * s["scale"]).masked_fill(hidden, -math.inf)
                lse[cu[b]:cu[b + 1], g] = torch.logsumexp(z, 1)
                out[cu[b]:cu[b + 1], g] = torch.softmax(z, 1) @ v
    return [out, lse]


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f32": 4, "f16": 2, "bf16": 2, "i32": 4}[case["dtype"]]
    if kind == "matmul":
        M, N, K = case["rows"], case["n"], case["k"]
        return {"bytes": N * K + M * K + M * N * size + (0 if case["dtype"] == "i32" else 4 * (M + N)), "flops": 2 * M * N * K}
    if kind == "prefix":
        n, lens = _lengths(case)
        pairs = sum(x * (y - (x - 1) / 2) for x, y in zip(n, lens))
        keys = case["prefix"] + sum(y - case["prefix"] for x, y in zip(n, lens) if x)
        rows = sum(n) * case["heads"]
        return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] + 2 * rows * case["dim"] * size + 4 * rows,
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    M, D = case["rows"], case["dim"]
    if kind == "quantise":
        return {"bytes": M * D * (size + 1) + 4 * M, "flops": 4 * M * D}
    # what is read and written of a whole tensor's size, and the vectors
    tensors = 2 + case["block"] + (case["gate"] == "token") + (not case["codes"])
    vectors = 1 + (case["norm"] == "layer") + (case["post"] != "none") + (case["gate"] == "channel")
    return {"bytes": (M * tensors + vectors) * D * size + (M * (D + 4) if case["codes"] else 0),
            "flops": M * D * (6 + 2 * case["block"] + 4 * (case["post"] != "none") + (case["gate"] != "none") + 3 * case["codes"])}
