"""The row operators' definitions in 64 bits, on the CPU, written apart from the library (tests only).

Quantities that the definition rounds to 32 bits are rounded here as well (both quotients of the quantizer and its
product, u = h * gain), everything else is 64-bit."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative
U32 = 2.0 ** -24


def f32(t):
    return t.float().double()


def edges(C, gs):
    step = C if gs == 0 or gs >= C else gs
    return [(lo, min(C, lo + step)) for lo in range(0, C, step)]


def quantize(v, gs):
    """Codes [rows][C], scales [rows][G] (both fp64) of 64-bit rows whose values fit 32 bits."""
    v = v.double().cpu()
    codes = torch.zeros_like(v)
    scales = torch.zeros((v.shape[0], len(edges(v.shape[1], gs))), dtype=torch.float64)
    for g, (lo, hi) in enumerate(edges(v.shape[1], gs)):
        part = v[:, lo:hi]
        finite = torch.isfinite(part).all(dim=1)
        amax = part.abs().nan_to_num(0.0, 0.0, 0.0).amax(dim=1)
        some = finite & (amax >= 1e-30)
        safe = torch.where(some, amax, torch.ones_like(amax))
        inv = f32(127.0 / safe)
        q = torch.round(f32(part.nan_to_num(0.0, 0.0, 0.0) * inv[:, None]))
        codes[:, lo:hi] = torch.where(some[:, None], q, torch.zeros_like(q))
        scale = torch.where(some, f32(safe / 127.0), torch.zeros_like(amax))
        scales[:, g] = torch.where(finite, scale, torch.full_like(scale, math.nan))
    return codes, scales


def spread(scales, C, gs):
    """Scales [rows][G] as [rows][C]."""
    out = torch.empty((scales.shape[0], C), dtype=torch.float64)
    for g, (lo, hi) in enumerate(edges(C, gs)):
        out[:, lo:hi] = scales[:, g:g + 1]
    return out


def rms_norm_quantize(x, residual, gain, eps, gs):
    """(stream in x's type, codes, scales)."""
    h = x.cpu() if residual is None else (x.cpu().float() + residual.cpu().float()).to(x.dtype)
    h64 = h.double()
    rstd = 1.0 / torch.sqrt((h64 * h64).mean(dim=1) + eps)
    codes, scales = quantize(f32(h64 * gain.double().cpu()), gs)
    return h, codes, scales * rstd[:, None]


def norm_scale_tolerance(C):
    """Relative error of a norm's scale: additions of C squares in any order that keeps partial sums of at most
    C / 32 + 40 terms in a row (half of it behind the square root), the products, and six more roundings."""
    return (0.5 * (C / 32 + 41) + 6) * U32


def activate(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def activation_error(z, act):
    """Error of the activation itself: SiLU is as exact as the fast exponential, 3 + |t| units in the last place; GELU
    has the error of 1 + erf, a few units in the last place of 1, times t / 2."""
    if act == "silu":
        return activate(z, act).abs() * (3.0 + z.abs()) * 2.0 ** -23
    if act == "gelu":
        return z.abs() * 2.0 ** -21
    return torch.zeros_like(z)


def linear(codes, scales, wcodes, wscales, gs, bias=None, act="none", gated=False, residual=None, dtype=torch.float32):
    """(y in 64 bits, largest error allowed) from codes and scales of both sides; weights [K] or, gated, [2K] rows."""
    C = codes.shape[1]
    groups = edges(C, gs)
    z = torch.zeros((codes.shape[0], wcodes.shape[0]), dtype=torch.float64)
    size = torch.zeros_like(z)
    unit = 16 if len(codes) <= 8 else 128              # channels that are summed in 32-bit integers at least
    for g, (lo, hi) in enumerate(groups):
        # A group may be summed in parts that begin and end at multiples of `unit` channels (several CTAs, or
        # several lanes for a few rows); each part is rounded on its own, and with s = a + b and a, b of opposite signs
        # |a| + |b| is any multiple of |s|.  So the size of a term is the sum of its smallest parts' magnitudes, which bounds the
        # magnitudes of any larger ones: |a + b| <= |a| + |b|.
        cuts = sorted({lo, hi} | set(range(-(-lo // unit) * unit, hi, unit)))
        for i, j in zip(cuts, cuts[1:]):
            t = (codes[:, i:j] @ wcodes[:, i:j].T) * scales[:, g:g + 1] * wscales[:, g][None]
            z += t
            size += t.abs()
    # per term: conversion and two products; then the additions: of a CTA's groups, or of a lane's parts, one in 32, and
    # eight between CTAs or warps, five between lanes
    err = size * (3 + max(len(groups), C / 512 + 1) + 13) * U32
    if bias is not None:
        z = z + bias.double().cpu()
        err = err + z.abs() * U32
    slope = 1.13                                       # of SiLU and GELU at most
    if gated:
        K = wcodes.shape[0] // 2
        a, v = z[:, :K], z[:, K:]
        fa = activate(a, act)
        ea = err[:, :K] * slope + activation_error(a, act) + 2 * U32 * fa.abs()
        y = fa * v
        err = ea * v.abs() + fa.abs() * err[:, K:] + ea * err[:, K:] + U32 * y.abs()
    else:
        y = activate(z, act)
        err = err * slope + activation_error(z, act) + 2 * U32 * y.abs()
    if residual is not None:
        y = y + residual.double().cpu()
        err = err + y.abs() * U32
    tiny = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[dtype]
    return y, err * (1 + 2.0 ** -8) + HALF[dtype] * y.abs() + tiny
