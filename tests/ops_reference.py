"""Plain 64-bit implementations of the operators around the V step, for their tests: torch on the
CPU in float64, straight from the formulas in include/pv.h, sharing nothing with the library."""
from __future__ import annotations

import math

import torch

EMAX = {"e2m1": 2, "e4m3": 8}
TOP = {"e2m1": 6.0, "e4m3": 448.0}
MANT = {"e2m1": 1, "e4m3": 3}
LOW = {"e2m1": 0, "e4m3": -6}           # exponent of the smallest normal value
# torch.finfo(t).eps / 2: the most that one rounding moves a value, relative to it
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def code_values(fmt):
    """The values of all codes, from their bits; NaN where the code is none."""
    m, bias, bits = MANT[fmt], {"e2m1": 1, "e4m3": 7}[fmt], {"e2m1": 4, "e4m3": 8}[fmt]
    out = []
    for c in range(1 << bits):
        sign = -1.0 if c >> (bits - 1) else 1.0
        e, f = c >> m & ((1 << (bits - 1 - m)) - 1), c & ((1 << m) - 1)
        v = math.ldexp(f, 1 - bias - m) if e == 0 else math.ldexp((1 << m) + f, e - bias - m)
        out.append(math.nan if fmt == "e4m3" and c & 0x7f == 0x7f else sign * v)
    return torch.tensor(out, dtype=torch.float64)


def split(codes, fmt):
    """One code an element."""
    c = codes.cpu().long()
    return torch.stack((c & 15, c >> 4), -1).flatten(-2) if fmt == "e2m1" else c


def decode(codes, scales, fmt, cols):
    v = code_values(fmt)[split(codes, fmt)]
    s = scales.cpu().long().repeat_interleave(32, 1)
    out = v * torch.pow(torch.tensor(2.0, dtype=torch.float64), (s - 127).double())
    out[s == 255] = math.nan
    return out[:, :cols]


def exponent(x):
    """floor(log2(x)) of positive float64 values."""
    return torch.frexp(x).exponent - 1


def quantize(x, fmt):
    """(codes, scales) of a matrix of finite or other values, in float64 arithmetic."""
    x = x.cpu().double()
    rows, cols = x.shape
    nblk = -(-cols // 32)
    x = torch.cat((x, torch.zeros(rows, nblk * 32 - cols, dtype=torch.float64)), 1).view(rows, nblk, 32)
    bad = ~torch.isfinite(x).all(2)
    x = torch.where(bad[:, :, None], 0.0, x)
    big = x.abs().amax(2)
    e = torch.where(big > 0, exponent(big) - EMAX[fmt], -127).clamp(-127, 127)
    v = x * torch.pow(torch.tensor(2.0, dtype=torch.float64), -e.double())[:, :, None]
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64),
                     (torch.where(v != 0, exponent(v.abs()), 0).clamp(min=LOW[fmt]) - MANT[fmt]).double())
    q = (torch.round(v / step) * step).clamp(-TOP[fmt], TOP[fmt])
    # the code of a magnitude is its place among the ascending magnitudes
    mags = code_values(fmt)[:128 if fmt == "e4m3" else 8]
    mags = mags[~torch.isnan(mags)]
    c = torch.searchsorted(mags, q.abs().contiguous())
    c = c + torch.where(torch.signbit(v), 128 if fmt == "e4m3" else 8, 0)
    c = torch.where(bad[:, :, None], 0, c).reshape(rows, nblk * 32)
    if fmt == "e2m1":
        c = c[:, 0::2] + 16 * c[:, 1::2]
    return c.to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


def rms_norm(x, residual, weight, eps, dtype):
    """(h as stored, rstd, y) in float64; h is rounded to `dtype` by way of the float32 sum."""
    h = x.cpu() if residual is None else (x.cpu().float() + residual.cpu().float()).to(dtype)
    h = h.double()
    rstd = (h.square().mean(1) + eps).rsqrt()
    return h, rstd, h * rstd[:, None] * weight.cpu().double()


def rms_norm_backward(dy, dh, h, weight, rstd):
    dy, h, w, r = dy.cpu().double(), h.cpu().double(), weight.cpu().double(), rstd.cpu().double()[:, None]
    n = h * r
    dx = r * (dy * w - n * (dy * w * n).mean(1, keepdim=True))
    if dh is not None:
        dx = dx + dh.cpu().double()
    return dx, (dy * n).sum(0)


def distill(logits, ids, top, t, weight=None):
    """(loss, lse, grad) in float64."""
    z, u, ids = logits.cpu().double() / t, top.cpu().double() / t, ids.cpu().long()
    R, V = z.shape
    w = torch.ones(R, dtype=torch.float64) if weight is None else weight.cpu().double()
    there = (ids >= 0) & (ids < V)
    at = torch.where(there, ids, 0)
    u = torch.where(there, u, -math.inf)
    any_ = (u > -math.inf).any(1) if ids.shape[1] else torch.zeros(R, dtype=torch.bool)
    # the largest logit first: a row of -3e38 leaves no digit of the sum's logarithm otherwise, in 64 bits neither
    largest = z.amax(1, keepdim=True)
    z = z - largest
    log_sum = torch.log(torch.exp(z).sum(1))
    lse = largest[:, 0] + log_sum
    if ids.shape[1]:
        log_p = torch.where(any_[:, None], u - torch.logsumexp(u, 1, keepdim=True), -math.inf)
    else:
        log_p = u
    p = torch.exp(log_p)
    log_q = z.gather(1, at) - log_sum[:, None]
    kl = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    target = torch.zeros(R, V, dtype=torch.float64).scatter_add(1, at, torch.where(there, p, 0.0))
    grad = t * (torch.exp(z - log_sum[:, None]) - target)
    on = (w != 0) & any_
    loss = torch.where(on, w * t * t * kl, 0.0)
    grad = torch.where(on[:, None], w[:, None] * grad, 0.0)
    return loss, torch.where(w != 0, lse, 0.0), grad


# half a step of the subnormal numbers
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def rounding(value, dtype):
    """The most that one rounding to `dtype` moves `value` (float64)."""
    return value.abs() * HALF_STEP[dtype] + TINY[dtype]


def check(got, want, allowed, what=""):
    """Every element within `allowed` of `want` (float64); NaN and infinities where `want` has them."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = (got - want).abs()[fine] - (allowed.double().expand(want.shape)[fine] if isinstance(allowed, torch.Tensor) else allowed)
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), int((off > 0).sum()))
