"""Plain 64-bit model of what a cache of keys and values retains, and causal attention behind it.

Shares no code with the library.  Everything stays on the device that it is given on; a low-precision row is kept as the values it
stands for in pask_prompt_attention, bf16(code * scale)."""
from __future__ import annotations

import math
import struct

import torch

DIM, GQA, GROUP = 128, 4, 32
RELEASE, LOW, HIGH = 0, 1, 2
LEVELS = {2: 1, 4: 7, 8: 127}
BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2       # 2^-8: a rounding to bf16 is off by at most this, relatively
F32_STEP = torch.finfo(torch.float32).eps                  # 2^-23


def blob(bits=4, window=0, n_layers=1):
    """A policy of three tags, tag a taking action a, in one layer group."""
    out = b"PASK" + struct.pack("<9I", 1, 3, 1, n_layers, 0, 65536, window, bits, GROUP) + b"\0" * (n_layers + -n_layers % 4)
    for a in (RELEASE, LOW, HIGH):
        out += struct.pack("<BBHff", a, 0, 0, 1.0, 1.0)
    return out


def stored_low(x, bits):
    """bf16 rows [n][heads][128] -> bf16 values of the format: scale fp16(amax / levels) and codes rint(x * (1 / scale)) in fp32, as the
    format says; the product of code and scale, exact in 64 bits, rounded once."""
    v = x.float().reshape(-1, GROUP)
    if not v.numel():
        return x
    a = v.abs().amax(1, keepdim=True)
    s = (a / torch.full_like(a, float(LEVELS[bits]))).clamp_max(65504.0).half().float()
    inv = torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))
    code = (v * inv).round().clamp(-LEVELS[bits], LEVELS[bits])
    return (code.double() * s.double()).to(torch.bfloat16).reshape(x.shape)


class Ref:
    """Per sequence: all tokens' keys, values and actions, in order of arrival."""

    def __init__(self, n_kv, bits, window):
        self.n_kv, self.bits, self.window, self.seqs = n_kv, bits, window, {}

    def append(self, seq, k, v, tags):
        old = self.seqs.get(seq)
        self.seqs[seq] = (k, v, tags) if old is None else tuple(torch.cat([a, b]) for a, b in zip(old, (k, v, tags)))

    def rows(self, seq):
        if seq not in self.seqs:
            e = torch.empty((0, self.n_kv, DIM), dtype=torch.bfloat16, device="cuda")
            return e, e
        k, v, tags = self.seqs[seq]
        recent = torch.arange(k.shape[0], device=k.device) >= k.shape[0] - self.window
        whole, low = recent | (tags == HIGH), ~recent & (tags == LOW)
        return tuple(torch.cat([x[whole], stored_low(x[low], self.bits)]) for x in (k, v))


def attend(q, k, v, hist):
    """q [n][heads][128], k, v [hist + n][kv][128]: token t sees keys 0 .. hist + t.  (out, lse, their tolerances) of an implementation that
    rounds the softmax weights and the result to bf16 and accumulates in 32 bits, keys in any number of parts that are joined."""
    n, m, scale = q.shape[0], k.shape[0], 1 / math.sqrt(DIM)
    out, lse = torch.empty(q.shape, dtype=torch.float64, device=q.device), torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    t_out, t_lse = torch.empty_like(out), torch.empty_like(lse)
    hidden = torch.arange(m, device=q.device)[None] > torch.arange(n, device=q.device)[:, None] + hist
    for h in range(q.shape[1]):
        a, b, c = q[:, h].double(), k[:, h // GQA].double(), v[:, h // GQA].double()
        s = (a @ b.T * scale).masked_fill(hidden, -math.inf)
        mag = (a.abs() @ b.abs().T).masked_fill(hidden, 0.0).amax(1) * scale
        l = torch.logsumexp(s, 1)
        p = torch.exp(s - l[:, None])
        o, absum = p @ c, p @ c.abs()
        # a score is a sum of 128 products in 32 bits (each addition off by at most a step of the running sum's bound), times the scale and
        # moved into powers of two (two more roundings); exp2 to 2 steps.  A weight is off by that, relatively, and so is their sum; then
        # one rounding of each weight to bf16, sums over m rows in 32 bits (16 more roundings for a row's parts), one of the result.
        eta = (mag * (DIM + 4) + s.masked_fill(hidden, 0.0).abs().amax(1) * 4) * F32_STEP + 8 * F32_STEP
        out[:, h], lse[:, h] = o, l
        t_out[:, h] = absum * (BF16_HALF_STEP + 2 * eta + (m + 16) * F32_STEP)[:, None] + o.abs() * BF16_HALF_STEP + 1e-30
        t_lse[:, h] = eta + (m + 16) * F32_STEP + l.abs() * 4 * F32_STEP
    return out, lse, t_out * 1.01, t_lse * 1.01


def check(out, lse, ref, where=""):
    o, l, to, tl = ref
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all()), f"{where}: not finite"
    d, e = (out.double() - o).abs() - to, (lse.double() - l).abs() - tl
    assert bool((d <= 0).all()), f"{where}: out off by {float((out.double() - o).abs().max()):.3g}, bound exceeded by {float(d.max()):.3g}"
    assert bool((e <= 0).all()), f"{where}: lse bound exceeded by {float(e.max()):.3g}"
