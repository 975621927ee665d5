"""Plain 64-bit model of latent caches: what each (sequence, layer) retains, and attention over it.

Shares no code with the library.  Rows are torch CPU tensors; low-precision rows are kept as the values they stand for.
"""
from __future__ import annotations

import math
import struct

import numpy as np
import torch

ROW, LATENT, GROUP = 576, 512, 32
RELEASE, LOW, HIGH = 0, 1, 2
LEVELS = {2: 1, 4: 7, 8: 127}
BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2       # 2^-8: a rounding to bf16 is off by at most this, relatively
F32_STEP = torch.finfo(torch.float32).eps                  # 2^-23


def blob(lut, n_layers, layer_group, low_bits=4, budget_q16=65536, floors=None):
    """A version-1 policy blob: lut[tag][group] actions."""
    n_tags, n_groups = len(lut), len(lut[0])
    out = b"PASK" + struct.pack("<9I", 1, n_tags, n_groups, n_layers, 0, budget_q16, 0, low_bits, 32)
    lg = bytes(layer_group)
    out += lg + b"\0" * (-len(lg) % 4)
    for z in range(n_tags):
        for g in range(n_groups):
            out += struct.pack("<BBHff", lut[z][g], 0 if floors is None else floors[z][g], 0, 1.0, 1.0)
    return out


def stored_low(x: torch.Tensor, bits: int) -> torch.Tensor:
    """bf16 rows [n][576] -> the bf16 values RETAIN-LOW stands for, in exact (64-bit) arithmetic."""
    v = x.double().reshape(-1, GROUP)
    s = (v.abs().amax(1, keepdim=True) / LEVELS[bits]).float().to(torch.bfloat16).double() if v.numel() else v[:, :1]
    s[s < 2.0 ** -126] = 0.0
    code = torch.where(s > 0, torch.round(v / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(v))
    assert code.numel() == 0 or code.abs().max() <= LEVELS[bits]
    return (code * s).to(torch.bfloat16).reshape(-1, ROW)


class Ref:
    def __init__(self, lut, layer_group, bits):
        self.lut, self.lg, self.bits = np.asarray(lut), layer_group, bits
        self.high, self.low = {}, {}

    def actions(self, layer, tags):
        lut = np.concatenate([self.lut[:, self.lg[layer]], np.full(256 - len(self.lut), HIGH)])
        return lut[np.asarray(tags)]

    def append(self, layer, seq, x, tags, actions=None):
        a = torch.from_numpy(self.actions(layer, tags) if actions is None else np.asarray(actions)).long()
        k = (layer, seq)
        empty = torch.empty((0, ROW), dtype=torch.bfloat16)
        self.high[k] = torch.cat([self.high.get(k, empty), x[a == HIGH]])
        self.low[k] = torch.cat([self.low.get(k, empty), stored_low(x[a == LOW], self.bits)])
        return a.to(torch.uint8)

    def reset(self, seq):
        for k in [k for k in self.high if k[1] == seq]:
            del self.high[k], self.low[k]

    def lens(self, layer, seq):
        k = (layer, seq)
        return [self.high[k].shape[0], self.low[k].shape[0]] if k in self.high else [0, 0]

    def rows(self, layer, seq):
        k = (layer, seq)
        return torch.cat([self.high[k], self.low[k]]) if k in self.high else torch.empty((0, ROW), dtype=torch.bfloat16)


def attend(q, k, v, scale, visible=None):
    """Softmax attention in 64 bits of q [h][d] (or [n][h][d] with visible [n]) on keys k [h or 1][m][d], values v [h or 1][m][e]:
    (out, lse, tolerance of out, tolerance of lse) of an implementation that rounds the softmax weights and the result to
    bf16 and accumulates in 32 bits."""
    q, k, v = q.double(), k.double(), v.double()
    m = k.shape[-2]
    if m == 0:
        o = torch.zeros(q.shape[:-1] + (v.shape[-1],), dtype=torch.float64)
        return o, torch.full(q.shape[:-1], -math.inf, dtype=torch.float64), torch.zeros_like(o), torch.zeros(q.shape[:-1], dtype=torch.float64)
    if visible is None:
        s, mag = torch.einsum("hd,hmd->hm", q, k.expand(q.shape[0], -1, -1)), torch.einsum("hd,hmd->hm", q.abs(), k.expand(q.shape[0], -1, -1).abs())
        vv = v.expand(q.shape[0], -1, -1)
        eq = "hm,hme->he"
    else:
        s, mag = torch.einsum("nhd,hmd->nhm", q, k), torch.einsum("nhd,hmd->nhm", q.abs(), k.abs())
        hidden = torch.arange(m)[None, :] >= visible[:, None]
        s = s.masked_fill(hidden[:, None, :], -math.inf)
        mag = mag.masked_fill(hidden[:, None, :], 0.0)
        vv, eq = v, "nhm,hme->nhe"
    s = s * scale
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.clamp_min(-1e300)[..., None])
    out, absum = torch.einsum(eq, p, vv), torch.einsum(eq, p, vv.abs())
    # a score is a sum of d products in 32 bits (each addition off by at most a step of the running sum's bound), times the
    # scale and moved into powers of two (two more roundings); exp2 to 2 steps.  A weight is off by that, relatively, and
    # so is their sum; then one rounding of each weight to bf16, the sum over m rows in 32 bits, one rounding of the result.
    # Scores that lie far below the row's largest weigh nothing: the bound uses each weight's own magnitude, so take the
    # largest |score| bound of the row.
    eta = (mag.amax(-1) * scale * (q.shape[-1] + 4) + s.masked_fill(s == -math.inf, 0.0).abs().amax(-1) * 4) * F32_STEP + 8 * F32_STEP
    t_out = absum * (BF16_HALF_STEP + 2 * eta + m * F32_STEP)[..., None] + out.abs() * BF16_HALF_STEP + 1e-30
    t_lse = eta + m * F32_STEP + lse.abs().clamp_max(1e30) * 4 * F32_STEP
    return out, lse, t_out * 1.01, t_lse * 1.01


def check(out, lse, ref, where=""):
    o, l, to, tl = ref
    out, lse = out.double().cpu(), lse.double().cpu()
    empty = l == -math.inf
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all()), f"{where}: rows with nothing to attend"
    assert bool(torch.isfinite(out).all()), f"{where}: not finite"
    d = (out - o).abs() - to
    d[empty] = 0.0
    assert bool((d <= 0).all()), f"{where}: out off by {float((out - o).abs().max()):.3g}, bound exceeded by {float(d.max()):.3g}"
    dl = torch.where(empty, torch.zeros_like(l), (lse - l).abs() - tl)
    assert bool((dl <= 0).all()), f"{where}: lse bound exceeded by {float(dl.max()):.3g}"
