"""The operators of a decoder layer in 8 bits by their definitions, on the CPU: in steps of 32 bits as they are defined bit for
bit, and by their formulas in 64 bits."""
import math

import torch

NONE, RMS, LAYER = 0, 1, 2


def codes_of(h):
    """(codes, scales) of float32 rows."""
    amax = h.abs().amax(1, keepdim=True)
    some = torch.isfinite(h).all(1, keepdim=True) & (amax >= 2.0 ** -100)
    safe = torch.where(some, amax, torch.ones_like(amax))
    full = torch.full_like(safe, 127.0)
    codes = torch.round(torch.where(some, h, torch.zeros_like(h)) * (full / safe)).to(torch.int8)
    zero = torch.isfinite(h).all(1, keepdim=True)
    scales = torch.where(some, safe / full, torch.where(zero, torch.zeros_like(safe), torch.full_like(safe, math.nan)))
    return codes, scales[:, 0]


def _steps(v, kind, gain, bias, eps):
    """float32 in and out; means in 64 bits."""
    if kind != NONE:
        wide = v.double()
        mean = wide.mean(1, keepdim=True) if kind == LAYER else torch.zeros(v.shape[0], 1, dtype=torch.float64)
        var = ((wide - mean) ** 2).mean(1, keepdim=True)
        eps = float(torch.tensor(eps, dtype=torch.float32))
        if kind == LAYER:
            v = v - mean.float()
        v = v * (1.0 / torch.sqrt(var + eps)).float()
    if gain is not None:
        v = v * gain.float()
    return v if bias is None else v + bias.float()


def norm_steps(x, z=None, *, norm=RMS, gain=None, bias=None, eps=1e-5, post_norm=NONE, post_gain=None, post_bias=None, gate=None, alpha=1.0):
    """(r, h in 32 bits)."""
    r = x.float() * torch.tensor(alpha, dtype=torch.float32)
    if z is not None:
        t = _steps(z.float(), post_norm, post_gain, post_bias, eps)
        r = r + (t if gate is None else gate.float() * t)
    r = r.to(x.dtype)
    return r, _steps(r.float(), norm, gain, bias, eps)


def norm_formula(v, kind, gain, bias, eps):
    """(h, size) in 64 bits: size is what the roundings of its steps are relative to."""
    v = v.double()
    eps = float(torch.tensor(eps, dtype=torch.float32))
    mean = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros(v.shape[0], 1, dtype=torch.float64)
    rstd = 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps) if kind != NONE else torch.ones_like(mean)
    g = 1.0 if gain is None else gain.double()
    b = 0.0 if bias is None else bias.double()
    h = (v - mean) * rstd * g + b
    return h, (v.abs() + 2 * mean.abs()) * rstd * abs(g) + abs(b)


def product(x, w, x_scales, w_scales, dtype):
    """Whole numbers below 2^53 at every step, then a rounding to 32 bits for each product with a scale."""
    sums = torch.matmul(x.double(), w.double().t().contiguous())
    if dtype == torch.int32:
        return sums.to(torch.int64).to(torch.int32)
    return (sums.to(torch.float32) * x_scales[:, None] * w_scales).to(dtype)
