"""The operators of quantised inference by their definitions, in 64 bits and one sequence, head and page after the other:
what the tests of the kernels compare with.  Works on CPU and GPU tensors alike."""
import math

import torch

EXP_MIN, EXP_MAX, EXP_NAN = -40, 40, -128


def need_of(a):
    """The smallest e in [-40, 40] with a <= 127 * 2^e, of a Python float."""
    if not math.isfinite(a):
        return EXP_NAN
    e = EXP_MIN
    while e < EXP_MAX and a > 127.0 * 2.0 ** e:
        e += 1
    return e


def append(k, v, k_exp, v_exp, k_new, v_new, cu, lens, table):
    """Returns the four arrays of the cache after the call (inputs are not modified)."""
    k, v, k_exp, v_exp = (t.clone() for t in (k, v, k_exp, v_exp))
    heads, T = k.shape[1], k.shape[2]
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        first = lens[b] - n
        for p in range(max(first, 0) // T, -(-lens[b] // T)):
            lo, hi = max(first, 0, p * T), min(lens[b], (p + 1) * T)
            if hi <= lo:
                continue
            page = table[b][p]
            for h in range(heads):
                for new, codes, exps in ((k_new, k[page, h], k_exp), (v_new, v[page, h].t(), v_exp)):
                    x = new[cu[b] + lo - first:cu[b] + hi - first, h].double()
                    need, held = need_of(float(x.abs().max()) if bool(torch.isfinite(x).all()) else math.inf), int(exps[page, h])
                    begins = lo == p * T
                    e = need if begins else EXP_NAN if EXP_NAN in (need, held) else max(need, held)
                    if begins:
                        codes.zero_()
                    elif e != EXP_NAN and e > held:
                        codes.copy_(torch.round(codes.double() * 2.0 ** (held - e)).to(torch.int8))
                    got = torch.zeros_like(x) if e == EXP_NAN else torch.round(x * 2.0 ** -e).clamp(-127, 127)
                    codes[lo - p * T:hi - p * T] = got.to(torch.int8)
                    exps[page, h] = e
    return k, v, k_exp, v_exp


def numbers(codes, exps, pages, h, across, length):
    """What a sequence's codes of a head stand for: (length, head_dim), NaN where a page's exponent says so."""
    c = codes[pages, h].double()
    if across:
        c = c.transpose(1, 2)
    e = exps[pages, h].double()
    scale = torch.where(e == EXP_NAN, torch.full_like(e, math.nan), torch.exp2(e))
    return (c * scale[:, None, None]).reshape(-1, c.shape[2])[:length]


def attention(k, v, k_exp, v_exp, q, cu, lens, table, scale, window=0):
    """(out, lse, size, score, weight): size is sum p |v| of each output, score and weight are scale * sum |q k| and p times
    the scale of its page of values at their largest for each row -- what the roundings of a computation in fewer bits are
    relative to."""
    rows, heads, d = q.shape
    H, T = k.shape[1], k.shape[2]
    G = heads // H
    q = q.double()
    out = torch.zeros(rows, heads, d, dtype=torch.float64, device=q.device)
    size = torch.zeros(rows, heads, d, dtype=torch.float64, device=q.device)
    score = torch.zeros(rows, heads, dtype=torch.float64, device=q.device)
    weight = torch.zeros(rows, heads, dtype=torch.float64, device=q.device)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(len(lens)):
        n, L = cu[b + 1] - cu[b], lens[b]
        if n == 0 or L == 0:
            continue
        pages = table[b][:-(-L // T)]
        for h in range(H):
            steps = torch.exp2(v_exp[pages, h].double()).repeat_interleave(T)
            kk, vv = numbers(k, k_exp, pages, h, False, L), numbers(v, v_exp, pages, h, True, L)
            for i in range(n):
                pos = L - n + i
                lo, hi = (max(0, pos - window + 1) if window else 0), pos + 1
                if hi <= lo:
                    continue
                qq = q[cu[b] + i, h * G:(h + 1) * G]
                s = qq @ kk[lo:hi].t().contiguous() * scale
                top = s.max(1, keepdim=True).values
                p = torch.exp(s - top)
                total = p.sum(1, keepdim=True)
                p = p / total
                at = slice(h * G, (h + 1) * G)
                out[cu[b] + i, at] = p @ vv[lo:hi]
                size[cu[b] + i, at] = p @ vv[lo:hi].abs()
                lse[cu[b] + i, at] = (top + torch.log(total))[:, 0]
                weight[cu[b] + i, at] = (p * steps[lo:hi]).max(1).values
                score[cu[b] + i, at] = (qq.abs() @ kk[lo:hi].t().abs().contiguous()).max(1).values * abs(scale)
    return out, lse, size, score, weight


def weights(codes, scales, group):
    """Integers c * scale, (n, k) int64."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(codes.shape[0], -1).long() - 8
    return c * scales.long().repeat_interleave(group, dim=1)[:, :c.shape[1]]


def order(row):
    """Indexes of a row's tokens: NaN first, then by larger value, among equals by lower index."""
    vals = row.tolist()
    return sorted(range(len(vals)), key=lambda i: (0 if math.isnan(vals[i]) else 1, -vals[i] if not math.isnan(vals[i]) else 0.0, i))


def logprobs(logits, targets, top):
    """Dict of lists, per row."""
    out = {"lse": [], "entropy": [], "target": [], "rank": [], "top_ids": [], "top": []}
    for r in range(logits.shape[0]):
        x = logits[r].double().cpu()
        first = order(x)
        vals = x.tolist()
        if any(math.isnan(t) for t in vals):
            lse = ent = math.nan
        elif max(vals) == -math.inf:
            lse, ent = -math.inf, 0.0
        elif max(vals) == math.inf:
            lse, ent = math.inf, math.nan
        else:
            m = max(vals)
            e = torch.exp(x - m)
            lse = m + math.log(float(e.sum()))
            p = e / e.sum()
            ent = float(-(p * torch.where(p > 0, torch.log(torch.where(p > 0, p, torch.ones_like(p))), torch.zeros_like(p))).sum())

        def logp(t):
            return -math.inf if lse == -math.inf else t - lse
        out["lse"].append(lse)
        out["entropy"].append(ent)
        t = int(targets[r])
        given = 0 <= t < len(vals)
        out["target"].append(logp(vals[t]) if given else math.nan)
        out["rank"].append(first.index(t) if given else -1)
        out["top_ids"].append(first[:top])
        out["top"].append([logp(vals[i]) for i in first[:top]])
    return out
