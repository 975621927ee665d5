"""Rotary positions in 64 bits: frequencies from their formulas, rotations as complex products."""
import math

import torch


def frequencies(rot, base=10000.0, scaling=0, factor=1.0, context=0.0, few=1.0, many=32.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        keep = 1.0
        if scaling == 1:
            keep = 0.0
        elif scaling == 2:
            keep = (context * f / (2 * math.pi) - few) / (many - few)
        elif scaling == 3:
            lo, hi = (rot * math.log(context / (r * 2 * math.pi)) / (2 * math.log(base)) for r in (many, few))
            lo, hi = max(0, math.floor(lo)), min(rot - 1, math.ceil(hi))
            keep = 1 - (i - lo) / max(hi - lo, 0.001)
        keep = min(1.0, max(0.0, keep))
        out.append(f * keep + f / factor * (1 - keep) if scaling else f)
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, pos, freq, interleaved=False, transpose=False, magnitude=1.0):
    """x [tokens][heads][dims] of any type: its rotation in 64 bits."""
    n = freq.numel()
    rot, y = 2 * n, x.double().clone()
    ang = pos.double()[:, None, None] * freq.to(x.device)
    turn = torch.polar(torch.full_like(ang, magnitude), -ang if transpose else ang)
    lo = y[..., 0:rot:2] if interleaved else y[..., :n]
    hi = y[..., 1:rot:2] if interleaved else y[..., n:rot]
    z = torch.complex(lo.contiguous(), hi.contiguous()) * turn
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        y[..., :n], y[..., n:rot] = z.real, z.imag
    return y


def bound(x, freq, interleaved, magnitude, dtype):
    """How far a result may be off, per element: fp32 arithmetic at an angle that is right to fp32, then half a step of the type.

    An angle goes to the sine as an fp32 number of half turns, at most 1 in magnitude: off by half a step, 2^-25 half turns, i.e. pi
    2^-25 < 2^-23 rad; sine and cosine (sincospi: 2 steps at most, magnitudes up to 1) by another 2 x 2^-23, the product with the
    magnitude by 2^-24.  A result a c - b s is then off by at most (|a| + |b|) magnitude times 2^-23 + 2^-22 + 2^-24 plus two roundings
    of 2^-24: under (|a| + |b|) magnitude 2^-21.  Then half a step of the result's type, or of its smallest subnormal number."""
    n = freq.numel()
    rot, y = 2 * n, x.double().abs()
    lo = y[..., 0:rot:2] if interleaved else y[..., :n]
    hi = y[..., 1:rot:2] if interleaved else y[..., n:rot]
    s = (lo + hi) * abs(magnitude)
    full = torch.zeros_like(y)
    if interleaved:
        full[..., 0:rot:2], full[..., 1:rot:2] = s, s
    else:
        full[..., :n], full[..., n:rot] = s, s
    fi = torch.finfo(dtype)
    return full * 2.0 ** -21 + (full > 0) * (full * fi.eps / 2 + fi.tiny * fi.eps / 2)
