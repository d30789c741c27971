"""Rotary positions and attention in 64 bits on the CPU, and how far results in
fewer bits may be from them.

``attend`` works row by row from the definition; ``Bound`` counts the roundings
of a computation in fp32 with results (and, for bf16 rows, weights) rounded to
the rows' type.
"""
from __future__ import annotations

import dataclasses
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # largest relative error of a rounding
F32 = HALF[torch.float32]


def rope(x, freqs, positions, interleaved=False, magnitude=1.0):
    """x [B, H, T, d] (any type), positions [B, T] -> fp64."""
    y = x.double().clone()
    R = freqs.numel()
    a = positions.double()[:, None, :, None] * freqs.double()
    c, s = magnitude * torch.cos(a), magnitude * torch.sin(a)
    i = torch.arange(R)
    p, r = (2 * i, 2 * i + 1) if interleaved else (i, i + R)
    u, w = x.double()[..., p], x.double()[..., r]
    y[..., p], y[..., r] = u * c - w * s, w * c + u * s
    return y


def rope_bound(x, freqs, out_dtype, interleaved=False, magnitude=1.0):
    """Largest |error| of each element: the angle's reduction (pi / 4 half steps),
    the series (two half steps), the factor, two products and their sum, one half step
    each, of |x1| + |x2|; then the result's own rounding."""
    R = freqs.numel()
    i = torch.arange(R)
    p, r = (2 * i, 2 * i + 1) if interleaved else (i, i + R)
    ax = x.double().abs()
    size = torch.zeros_like(ax)
    size[..., p] = size[..., r] = (ax[..., p] + ax[..., r]) * abs(magnitude)
    # bf16 results: half a step of a value of at most `size`
    return size * 8 * F32 + (0 if out_dtype == torch.float32 else torch.maximum(size, ax) * HALF[out_dtype])


@dataclasses.dataclass
class Row:
    out: torch.Tensor    # [d] fp64
    bound: torch.Tensor  # [d] largest |error|


def attend(q, K, V, dist, allowed, scale, softcap=0.0, slope=0.0, row_dtype=torch.float32):
    """One query row q [d] over K, V [n, d]; dist [n] distances, allowed [n].

    ``row_dtype``: type of the rows; bf16 with fp32 queries (three bf16 terms)
    counts as fp32, bf16 queries and results as bf16."""
    j = torch.nonzero(allowed).flatten()
    d = q.numel()
    if j.numel() == 0:
        return Row(torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64))
    q, K, V = q.double(), K[j].double(), V[j].double()
    raw = K @ q * scale
    s = softcap * torch.tanh(raw / softcap) if softcap else raw
    s = s - slope * dist[j].double()
    p = torch.softmax(s, 0)
    out = p @ V
    # errors of a score: d products and sums and the scale, the cap (its argument's
    # error shrinks by the slope of tanh; tanh itself is within 2^-22 of 1), the
    # bias, and the difference to the row's maximum in units of log 2
    mag = (K.abs() @ q.abs() * scale)
    delta = mag * (d + 4) * F32
    if softcap:
        delta = delta + softcap * 2.0 ** -22 + s.abs() * 4 * F32
    delta = delta + (slope * dist[j].double()) * 4 * F32 + (s.abs() + s.abs().max()) * 4 * F32
    delta = float(delta.max())
    n = j.numel()
    w = (2 * math.expm1(2 * delta)          # weights and their sum
         + 2 * (n + 64) * F32               # both sums, joins of parts, the division
         + (HALF[torch.bfloat16] if row_dtype == torch.bfloat16 else 2 * F32))
    bound = (p @ V.abs()) * w + out.abs() * HALF[row_dtype]
    return Row(out, bound)
